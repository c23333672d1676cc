"""Chunk steps that make a workgroup's waves take a KV head each, look up more pages than fit one
look-up, and walk several wide row tiles, against float64 (which step does what: chunk_regimes.py).

The tolerance is that of test_gpu_block_chunk.py, with its bound on logits taken from the inputs: a
logit is an fp32 sum of 128 products, off by 2^-24 x 128 x sum |q k| scale at most, and sum |q k|
scale is below 2^5 here (normal queries and keys, 128 of them: 128 x 0.64 x 0.088 = 7.2 expected).
That is 2^-12, and enters twice: 2^-11 A.  A row tile's sums over many parts are joined in fp32."""
import pytest

from chunk_regimes import STEPS, max_context

pytestmark = pytest.mark.gpu
D, N = 128, 64


def _cache(hq, hkv, held, T, mc, seed):
    """A cache of few pages that all blocks take in turn (a step only reads them)."""
    import paper_2608_05326_amd as qv
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pages = 37
    bc = qv.BlockCache(qv.BlockConfig(len(held), hq, hkv, mc, num_pages=pages, chunk_tokens=T))
    for name in ("k_codes", "v_codes"):
        x = getattr(bc, name)
        x.copy_(torch.randn(x.shape, generator=g, device="cuda").mul_(35).clamp_(-127, 127).round_())
    for name in ("k_scale", "v_scale"):
        x = getattr(bc, name)
        x.copy_((0.5 + torch.rand(x.shape, generator=g, device="cuda")) / 35)
    for name in ("k_tail", "v_tail"):
        x = getattr(bc, name)
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    bc.table = torch.randint(0, pages, bc.table.shape, generator=g, device="cuda").to(torch.int32)
    bc.lens = torch.tensor(held, dtype=torch.int32)
    return bc, g


def _check_place(bc, s, held, n, q, k, v, out):
    """q, out [n, H_q, d], k, v [n, H_kv, d] of place s, one KV head at a time."""
    import torch
    c = bc.cfg
    G, blocks = c.num_q_heads // c.num_kv_heads, held // N
    p = bc.table[s, :blocks].long()
    for h in range(c.num_kv_heads):
        kk = (bc.k_codes[0, p, h].double() * bc.k_scale[0, p, h].double()[:, None, None]).reshape(-1, D)
        vv = (bc.v_codes[0, p, h].double() * bc.v_scale[0, p, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)
        kk = torch.cat([kk, bc.k_tail[0, s, h, :held % N].double(), k[:, h].double()]).t().contiguous()
        vv = torch.cat([vv, bc.v_tail[0, s, h, :held % N].double(), v[:, h].double()])
        va = vv.abs()
        step = max(1, (1 << 27) // (G * (held + n)))
        for r in range(0, n, step):
            e = min(r + step, n)
            x = q[r:e, h * G:h * G + G].double().reshape(-1, D)
            w = (x @ kk[:, :held + e].contiguous()) * D ** -0.5
            seen = torch.arange(held + e, device="cuda")[None] <= torch.arange(held + r, held + e, device="cuda")[:, None]
            w.view(e - r, G, held + e).masked_fill_(~seen[:, None], -torch.inf)
            w = torch.softmax(w, 1)
            o, A = w @ vv[:held + e], w @ va[:held + e]
            tol = 2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A
            err = (out[r:e, h * G:h * G + G].double().reshape(-1, D) - o).abs()
            assert bool((err <= tol).all()), (s, h, r, (err / tol).max().item())


@pytest.mark.parametrize("name", STEPS)
def test_step(name):
    import torch
    hq, hkv, held, lens, _ = STEPS[name]
    T = sum(lens)
    bc, g = _cache(hq, hkv, held, T, max_context(held, lens), seed=len(name))
    q, k, v = (torch.randn(T, h, D, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    out = torch.full_like(q, 7.0)
    cu = torch.tensor([sum(lens[:s]) for s in range(len(lens) + 1)], dtype=torch.int32).cuda()
    bc.chunk_workspace.fill_(0xff)
    bc.attend_chunk(0, q, k, v, cu, out)
    again = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, cu, again)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    at = 0
    for s, (a, n) in enumerate(zip(held, lens)):
        rows = slice(at, at + n)
        at += n
        if a < 0:
            assert bool((out[rows] == 7.0).all())
        elif n:
            _check_place(bc, s, a, n, q[rows], k[rows], v[rows], out[rows])
