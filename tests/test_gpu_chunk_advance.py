"""Chunk steps whose bounds lie outside the packed rows, end to end: what is held afterwards, and a
step that follows, are those of the same step with bounds that lie inside."""
import pytest

from test_gpu_block_chunk import _cache, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counted", [False, True])
def test_bounds_outside_the_rows(counted):
    import torch
    held, T = [10, 64, 3], 224
    outside, inside = ([-5, 60, 124, 1 << 30], [0, 60, 124, 224])
    counts = torch.tensor([7, 1 << 30, 99], dtype=torch.int32).cuda() if counted else None
    caches = [_cache(held, 4, 2, T, seed=80, extra=400, fill=0.0) for _ in range(2)]
    q, k, v = _rows(T, 4, 2, seed=81)
    outs = []
    for bc, bounds in zip(caches, (outside, inside)):
        cu = torch.tensor(bounds, dtype=torch.int32).cuda()
        got = []
        for _ in range(2):
            out = torch.full_like(q, 7.0)
            bc.attend_chunk(0, q, k, v, cu, out)
            bc.append(0, k, v, cu, counts=counts)
            bc.advance(cu, counts, total_tokens=T)
            got += [out, bc.lens.clone()]
        outs.append(got)
    first = [7, 64, 99] if counted else [60, 64, 100]
    assert outs[0][1].tolist() == [a + n for a, n in zip(held, first)]
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name
