"""Chunk attention over the whole range of softmax scales and of queries, against float64.

The tolerance is that of test_gpu_block_chunk.py: it has no term for the scale, since a logit's
error is relative to sum |q k| scale, which stays as there."""
import pytest

from test_gpu_block_chunk import D, N, _cache, _check, _cu, _rows
from test_gpu_block_cache import _bf16

pytestmark = pytest.mark.gpu

LENS = [[5, 3], [60, 2], [300, 260]]     # 32, 64 and 256 rows a workgroup


def _scaled(base, scale, chunk):
    """The cache `base` with a softmax scale of its own."""
    import paper_2608_05326_amd as qv
    c = base.cfg
    bc = qv.BlockCache(qv.BlockConfig(c.batch, c.num_q_heads, c.num_kv_heads, c.max_context, num_pages=base.num_pages,
                                      softmax_scale=scale, chunk_tokens=chunk))
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "lens"):
        setattr(bc, name, getattr(base, name))
    return bc


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("log_scale", [-64, -50, -45, -44])
def test_small_queries_at_small_scales(lens, log_scale):
    """Rows of zeros, of bf16's smallest values and of small ones beside ordinary rows: logits
    next to zero, every key that a row sees weighs about the same, masked ones nothing."""
    import torch
    held, T = [200, 77], sum(lens)
    scale = 2.0 ** log_scale
    bc = _scaled(_cache(held, 4, 2, T, seed=70, extra=400), scale, T)
    q, k, v = _rows(T, 4, 2, seed=71)
    small = torch.tensor([0.0, 2.0 ** -133, 2.0 ** -120, 2.0 ** -106, 2.0 ** -90, 1.0], device="cuda")
    kind = torch.arange(T * 4, device="cuda").view(T, 4, 1) % 6
    tiny = torch.where(kind == 1, torch.randint(-3, 4, q.shape, device="cuda").double(), q.double())
    q = (tiny * small[kind].double()).float().bfloat16()
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    _check(bc, held, lens, q, k, v, out, scale=scale)


@pytest.mark.parametrize("lens", LENS, ids=str)
def test_small_queries_beside_large_keys_at_small_scales(lens):
    """Logits of ordinary size from the smallest scale: keys of 2^115, queries of 2^-51 to 2^-60."""
    import torch
    held, T, scale = [40, 33], sum(lens), 2.0 ** -64
    bc = _scaled(_cache(held, 4, 2, T, seed=72, extra=400), scale, T)
    bc.k_tail.copy_((bc.k_tail.float() * 2.0 ** 115).bfloat16())
    for e in (-51, -60):
        q, k, v = _rows(T, 4, 2, seed=73)
        q, k = (q.float() * 2.0 ** e).bfloat16(), (k.float() * 2.0 ** 115).bfloat16()
        out = torch.full_like(q, 7.0)
        bc.attend_chunk(0, q, k, v, _cu(lens), out)
        _check(bc, held, lens, q, k, v, out, scale=scale)


def _keys(shape, e, seed):
    """+-[1, 2) 2^e in bf16: no subnormal numbers among small keys."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = 1.0 + torch.rand(*shape, generator=g) * 0.99
    return (x * (torch.randint(0, 2, shape, generator=g) * 2 - 1) * 2.0 ** e).bfloat16().cuda()


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("log_scale,e,pages", [(-3.5, 112, True), (-3.5, 120, True), (-3.5, 124, False), (64, 0, True),
                                               (64, 40, True), (64, 59, False), (10, 90, True)])
def test_large_queries_beside_small_keys(lens, log_scale, e, pages):
    """Logits of ordinary size from queries of 2^e: keys as much smaller, past the scale as well."""
    import torch
    held = [200, 77] if pages else [40, 33]
    T, scale = sum(lens), 2.0 ** log_scale
    down = -e if log_scale < 0 else -e - log_scale
    bc = _scaled(_cache(held, 4, 2, T, seed=74, extra=400, fill=0.0), scale, T)
    bc.k_scale *= 2.0 ** down
    bc.k_tail.copy_(_keys(bc.k_tail.shape, down, seed=75))
    q, _, v = _rows(T, 4, 2, seed=76)
    q = (q.float().clamp(-4, 4) * 2.0 ** (e - 2)).bfloat16()
    k = _keys(v.shape, down, seed=77)
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    _check(bc, held, lens, q, k, v, out, scale=scale)


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("log_s", [-80, -81, -100])
def test_values_of_the_smallest_scales(lens, log_s):
    """Weights are rounded with their block's value scale s in them: one below 2^-126 / s of the row's
    largest may count as zero, which n keys bring to n 2^-126 / s max |v|.  Queries of 4: sum |q k|
    scale below 2^6, a logit off by 2^-24 x 128 x 2^6 = 2^-11, twice."""
    import torch
    held, T, s = [6400, 130], sum(lens), 2.0 ** log_s
    bc = _cache(held, 4, 2, T, seed=78, extra=400, fill=0.0)
    bc.v_scale.fill_(s)
    bc.v_tail.copy_(bc.v_tail.float() * (32 * s))
    q, k, v = _rows(T, 4, 2, seed=79, scale=4.0)
    v = (v.float() * (32 * s)).bfloat16()
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    at = 0
    for p, (a, n) in enumerate(zip(held, lens)):
        pages = bc.table[p, :a // N].long()
        mask = torch.arange(a + n, device="cuda")[None] <= torch.arange(a, a + n, device="cuda")[:, None]
        for h in range(4):
            g = h // 2
            kk = (bc.k_codes[0, pages, g].double() * bc.k_scale[0, pages, g].double()[:, None, None]).reshape(-1, D)
            vv = (bc.v_codes[0, pages, g].double() * s).transpose(1, 2).reshape(-1, D)
            kk = torch.cat([kk, bc.k_tail[0, p, g, :a % N].double(), k[at:at + n, g].double()])
            vv = torch.cat([vv, bc.v_tail[0, p, g, :a % N].double(), v[at:at + n, g].double()])
            w = q[at:at + n, h].double() @ kk.t().contiguous() * D ** -0.5
            w = torch.softmax(torch.where(mask, w, -torch.inf), 1)
            o, A = w @ vv, w @ vv.abs()
            tol = 2.0 ** -8 * (A + o.abs()) + 2.0 ** -10 * A + (a + n) * 2.0 ** -126 / s * vv.abs().max()
            err = (out[at:at + n, h].double() - o).abs()
            assert bool((err <= tol).all()), (p, h, (err / tol).max().item())
        at += n
