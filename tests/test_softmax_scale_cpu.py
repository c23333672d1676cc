"""The softmax scales that the packed-prompt and block-cache calls take: 0 (the default) or
2^-64 .. 2^64.  Outside, scale log2 e is no normal float or logits of ordinary size need
products q k past fp32's range."""
import ctypes

import pytest

import paper_2608_05326_amd as qv
from paper_2608_05326_amd import qevict as m


def _status(scale):
    """Of a prompt call with nothing to do and of a block cache's workspace size."""
    lib = qv.load_library()
    p = m._PromptConfig(m.ABI_VERSION, 1, 0, 8, 2, 128, scale, 1024, 128, 256, 128, 256, 128, 1024, 128)
    b = m._BlockConfig(m.ABI_VERSION, 2, 8, 2, 128, 1000, 40, scale)
    n = ctypes.c_size_t()
    return (lib.qevict_prompt_attend(ctypes.byref(p), None, None, None, None, None, None),
            lib.qevict_block_workspace_size(ctypes.byref(b), ctypes.byref(n)))


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -64, 1e-3, 128 ** -0.5, 1.0, 2.0 ** 64])
def test_taken(scale):
    assert _status(scale) == (m.OK, m.OK)


@pytest.mark.parametrize("scale", [1e-45, 1e-38, 2.0 ** -65, 2.0 ** 64 * 1.5, 2.4e38, 3.4e38, -0.1])
def test_refused(scale):
    assert _status(scale) == (m.ERR_INVALID_ARG, m.ERR_INVALID_ARG)
    assert b"softmax_scale" in qv.load_library().qevict_last_error()
