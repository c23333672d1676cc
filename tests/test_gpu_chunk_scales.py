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
