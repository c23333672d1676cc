"""Sizes that do not fit the C ABI's 32-bit fields are refused instead of being cut to their
low bits (decided before anything touches a device)."""
import pytest
import torch

import paper_2608_05326_amd as qv
from paper_2608_05326_amd import qevict as m


@pytest.mark.parametrize("kw", [
    dict(max_context=(1 << 32) + 64, num_pages=4), dict(batch=(1 << 32) + 1, num_pages=4),
    dict(num_pages=(1 << 32) + 4), dict(num_q_heads=(1 << 32) + 2), dict(num_kv_heads=(1 << 32) + 1),
    dict(head_dim=(1 << 32) + 128), dict(max_context=1 << 31)])
def test_block_config(kw):
    cfg = dict(batch=1, num_q_heads=2, num_kv_heads=1, max_context=64)
    cfg.update(kw)
    with pytest.raises(ValueError, match="2\\^31"):
        qv.BlockCache(qv.BlockConfig(**cfg))


class Rows:
    """A packed tensor's description (rows that repeat one: a stride of 0)."""
    dtype = torch.bfloat16

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def get_device(self):
        return 0

    def stride(self):
        return 0, 128, 1

    def data_ptr(self):
        return 1 << 20


@pytest.mark.parametrize("shape", [((1 << 32) + 100, 2, 128), (100, (1 << 32) + 2, 128), (1 << 31, 2, 128)])
def test_packed_rows(shape):
    assert m._rows(Rows(100, 2, 128), torch, 0, "k") == (1 << 20, 0, 128)
    with pytest.raises(ValueError, match="2\\^31"):
        m._rows(Rows(*shape), torch, 0, "k")


def test_bounds():
    class Bounds(Rows):
        dtype = torch.int32

        def dim(self):
            return 1

        def is_contiguous(self):
            return True
    n = (1 << 32) + 3
    with pytest.raises(ValueError, match="2\\^31"):
        m._int32(Bounds(n), torch, 0, "cu_tokens", n)
