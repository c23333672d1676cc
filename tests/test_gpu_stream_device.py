"""A stream has to belong to the device of the tensors: a kernel launched on another device's
stream would read addresses that are not that device's.  Refused on the host."""
import pytest

pytestmark = pytest.mark.gpu
D = 128


class Elsewhere:
    """A stream that says that it is another device's."""

    def __init__(self, st):
        import torch
        self.device, self.cuda_stream = torch.device("cuda", st.device.index + 1), st.cuda_stream


def test_prompt_attend_refuses_a_stream_of_another_device():
    import torch
    import paper_2608_05326_amd as qv
    q = torch.zeros(4, 2, D, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    st = torch.cuda.Stream()
    with pytest.raises(ValueError):
        qv.prompt_attend(q, q, q, cu, out, stream=Elsewhere(st))
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    qv.prompt_attend(q, q, q, cu, out, stream=st)
    torch.cuda.synchronize()
    assert bool((out == 0.0).all())


def test_a_cache_refuses_a_stream_of_another_device():
    import torch
    import paper_2608_05326_amd as qv
    with pytest.raises(ValueError):
        qv.BlockCache(qv.BlockConfig(1, 2, 1, 64), stream=Elsewhere(torch.cuda.Stream()))
