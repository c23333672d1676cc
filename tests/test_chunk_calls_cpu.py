"""Host-side refusals of the rotation, append and chunk-attention calls, the rotation's object
and advance(): everything that is decided before a device is touched (pointers are never
followed)."""
import ctypes
import math

import pytest
import torch

import paper_2608_05326_amd as qv
from paper_2608_05326_amd import qevict as m

P = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 8)
BYTE = ctypes.c_void_p((1 << 20) + 2)


def _rotary(**kw):
    c = m._Rotary(m.ABI_VERSION, 64, 3, 0)
    for n, x in kw.items():
        if n == "axis":
            c.axis[x[0]] = x[1]
        else:
            setattr(c, n, x)
    return c


def _rotate(rot=None, pos=P, q=P, k=P, qo=P, ko=P, **kw):
    c = m._RotateConfig(m.ABI_VERSION, 100, 8, 2, 128, 0, 3, 1, 1024, 128, 256, 128, 1024, 128, 256, 128)
    for n, x in kw.items():
        setattr(c, n, x)
    rot = _rotary() if rot is None else rot
    return qv.load_library().qevict_rotate(ctypes.byref(c), ctypes.byref(rot), pos, q, k, qo, ko, None)


BAD_ROTARY = [
    (dict(abi_version=3), m.ERR_UNSUPPORTED),
    (dict(num_pairs=0), m.ERR_UNSUPPORTED),
    (dict(num_pairs=12), m.ERR_UNSUPPORTED),
    (dict(num_pairs=72), m.ERR_UNSUPPORTED),
    (dict(num_axes=0), m.ERR_UNSUPPORTED),
    (dict(num_axes=5), m.ERR_UNSUPPORTED),
    (dict(interleaved=2), m.ERR_INVALID_ARG),
    (dict(axis=(17, 3)), m.ERR_INVALID_ARG),
]


@pytest.mark.parametrize("kw,status", BAD_ROTARY)
def test_rotate_refuses_the_rotation(kw, status):
    assert _rotate(_rotary(**kw)) == status
    assert qv.load_library().qevict_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=5), m.ERR_UNSUPPORTED),
    (dict(head_dim=64), m.ERR_UNSUPPORTED),
    (dict(num_q_heads=0), m.ERR_INVALID_ARG),
    (dict(num_k_heads=-1), m.ERR_INVALID_ARG),
    (dict(inverse=2), m.ERR_INVALID_ARG),
    (dict(total_tokens=-1), m.ERR_INVALID_ARG),
    (dict(pos=None), m.ERR_INVALID_ARG),
    (dict(pos=BYTE), m.ERR_INVALID_ARG),
    (dict(position_token_stride=-1), m.ERR_INVALID_ARG),
    (dict(position_axis_stride=-3), m.ERR_INVALID_ARG),
    (dict(position_token_stride=1 << 60), m.ERR_INVALID_ARG),
    (dict(q=None), m.ERR_INVALID_ARG),
    (dict(qo=ODD), m.ERR_INVALID_ARG),
    (dict(k=ODD), m.ERR_INVALID_ARG),
    (dict(ko=None), m.ERR_INVALID_ARG),
    (dict(q_token_stride=-8), m.ERR_INVALID_ARG),
    (dict(k_head_stride=12), m.ERR_INVALID_ARG),
    (dict(q_out_token_stride=512), m.ERR_INVALID_ARG),       # rows overlap
    (dict(k_out_head_stride=0), m.ERR_INVALID_ARG),
    (dict(q_token_stride=2048), m.ERR_INVALID_ARG),          # in place with other strides
    (dict(total_tokens=1 << 28), m.ERR_UNSUPPORTED),
])
def test_rotate_refuses(kw, status):
    assert _rotate(**kw) == status
    assert qv.load_library().qevict_last_error()


def test_nothing_to_rotate_is_ok():
    assert _rotate(total_tokens=0, pos=None, q=None, k=None, qo=None, ko=None) == m.OK


def _block(call, cfg=None, layer=None, rot=None, rows=None, **kw):
    lib = qv.load_library()
    c = m._BlockConfig(m.ABI_VERSION, 2, 8, 2, 128, 1000, 40, 0.0)
    for n, x in (cfg or {}).items():
        setattr(c, n, x)
    p = m._BlockLayer(*[1 << 20] * 8)
    for n, x in (layer or {}).items():
        setattr(p, n, x)
    if call == "chunk":
        r = m._ChunkConfig(m.ABI_VERSION, 100, 1024, 128, 256, 128, 256, 128, 1024, 128)
        for n, x in (rows or {}).items():
            setattr(r, n, x)
        a = dict(q=P, k=P, v=P, cu=P, out=P, ws=P, size=1 << 40)
        a.update(kw)
        return lib.qevict_block_attend_chunk(ctypes.byref(c), ctypes.byref(p), ctypes.byref(r), a["q"], a["k"],
                                             a["v"], a["cu"], a["out"], a["ws"], a["size"], None)
    a = dict(k=P, k_st=256, k_sh=128, v=P, v_st=256, v_sh=128, cu=P, counts=None, total=100, pos=P, p_st=3, p_sa=1)
    a.update(kw)
    return lib.qevict_block_append(ctypes.byref(c), ctypes.byref(p), a["k"], a["k_st"], a["k_sh"], a["v"],
                                   a["v_st"], a["v_sh"], a["cu"], a["counts"], a["total"],
                                   None if rot is None else ctypes.byref(rot), a["pos"], a["p_st"], a["p_sa"], None)


@pytest.mark.parametrize("call", ["append", "chunk"])
@pytest.mark.parametrize("cfg,layer,status", [
    (dict(abi_version=5), {}, m.ERR_UNSUPPORTED),
    (dict(head_dim=96), {}, m.ERR_UNSUPPORTED),
    (dict(num_q_heads=34), {}, m.ERR_UNSUPPORTED),          # 17 heads per KV head
    (dict(num_q_heads=7), {}, m.ERR_INVALID_ARG),
    (dict(batch=0), {}, m.ERR_INVALID_ARG),
    (dict(max_context=(1 << 30) + 1), {}, m.ERR_UNSUPPORTED),
    (dict(num_pages=-1), {}, m.ERR_INVALID_ARG),
    (dict(batch=1 << 24), {}, m.ERR_UNSUPPORTED),
    (dict(softmax_scale=-0.5), {}, m.ERR_INVALID_ARG),
    ({}, dict(k_codes=0), m.ERR_INVALID_ARG),
    ({}, dict(v_tail=(1 << 20) + 2), m.ERR_INVALID_ARG),
    ({}, dict(lens=(1 << 20) + 1), m.ERR_INVALID_ARG),
])
def test_block_calls_refuse(call, cfg, layer, status):
    assert _block(call, cfg, layer) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), m.ERR_INVALID_ARG),
    (dict(v=ODD), m.ERR_INVALID_ARG),
    (dict(k_st=-256), m.ERR_INVALID_ARG),
    (dict(v_sh=4), m.ERR_INVALID_ARG),
    (dict(cu=None), m.ERR_INVALID_ARG),
    (dict(counts=BYTE), m.ERR_INVALID_ARG),
    (dict(total=-1), m.ERR_INVALID_ARG),
    (dict(rot=_rotary(), pos=None), m.ERR_INVALID_ARG),
    (dict(rot=_rotary(), p_st=-1), m.ERR_INVALID_ARG),
    (dict(total=1 << 30), m.ERR_UNSUPPORTED),
] + [(dict(rot=_rotary(**kw)), status) for kw, status in BAD_ROTARY])
def test_append_refuses(kw, status):
    assert _block("append", **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), m.ERR_INVALID_ARG),
    (dict(k=ODD), m.ERR_INVALID_ARG),
    (dict(v=None), m.ERR_INVALID_ARG),
    (dict(out=ODD), m.ERR_INVALID_ARG),
    (dict(cu=None), m.ERR_INVALID_ARG),
    (dict(cu=BYTE), m.ERR_INVALID_ARG),
    (dict(ws=None), m.ERR_WORKSPACE),
    (dict(ws=ODD), m.ERR_WORKSPACE),
    (dict(size=0), m.ERR_WORKSPACE),
    (dict(rows=dict(abi_version=3)), m.ERR_UNSUPPORTED),
    (dict(rows=dict(total_tokens=-1)), m.ERR_INVALID_ARG),
    (dict(rows=dict(total_tokens=1 << 28)), m.ERR_UNSUPPORTED),
    (dict(rows=dict(q_token_stride=-8)), m.ERR_INVALID_ARG),
    (dict(rows=dict(v_head_stride=4)), m.ERR_INVALID_ARG),
    (dict(rows=dict(k_token_stride=1 << 23)), m.ERR_UNSUPPORTED),
    (dict(rows=dict(v_token_stride=1 << 24)), m.ERR_UNSUPPORTED),
    (dict(rows=dict(out_token_stride=512)), m.ERR_INVALID_ARG),
])
def test_attend_chunk_refuses(kw, status):
    assert _block("chunk", **kw) == status


def test_nothing_to_do_is_ok():
    assert _block("append", total=0, k=None, v=None, cu=None) == m.OK
    assert _block("chunk", rows=dict(total_tokens=0), q=None, k=None, v=None, out=None, ws=None) == m.OK


def test_chunk_workspace_size():
    lib = qv.load_library()
    c = m._BlockConfig(m.ABI_VERSION, 2, 8, 2, 128, 1000, 40, 0.0)
    n = ctypes.c_size_t()
    sizes = []
    for total in (0, 1, 8, 100, 1 << 20):
        assert lib.qevict_block_chunk_workspace_size(ctypes.byref(c), total, ctypes.byref(n)) == m.OK
        sizes.append(n.value)
    assert sizes[0] == 0 and sizes == sorted(sizes) and sizes[1] > 0
    lib.qevict_block_chunk_workspace_size(ctypes.byref(c), 100, ctypes.byref(n))
    assert _block("chunk", size=n.value - 1) == m.ERR_WORKSPACE
    assert lib.qevict_block_chunk_workspace_size(ctypes.byref(c), -1, ctypes.byref(n)) == m.ERR_INVALID_ARG
    assert lib.qevict_block_chunk_workspace_size(ctypes.byref(c), 1 << 28, ctypes.byref(n)) == m.ERR_UNSUPPORTED
    assert lib.qevict_block_chunk_workspace_size(ctypes.byref(c), 100, None) == m.ERR_INVALID_ARG
    assert lib.qevict_block_chunk_workspace_size(None, 100, ctypes.byref(n)) == m.ERR_INVALID_ARG


# ------------------------------------------------------------ the rotation's object
@pytest.mark.parametrize("kw", [
    dict(dim=0), dict(dim=24), dict(dim=144), dict(base=0.0), dict(base=float("nan")), dict(base=-3.0),
    dict(sections=(64, 64)), dict(sections=(65, -1)), dict(sections=(16,) * 5, dim=128),
    dict(sections=(64,), axes=[0] * 64), dict(axes=[0] * 63), dict(axes=[4] * 64), dict(axes=[-1] + [0] * 63),
    dict(inv_freq=[1.0] * 63), dict(inv_freq=[float("inf")] * 64), dict(inv_freq=[2.0 ** 33] * 64),
])
def test_rotary_refuses(kw):
    with pytest.raises(ValueError):
        qv.Rotary(**kw)


def test_rotary_holds_turns():
    r = qv.Rotary(base=10000.0, sections=(16, 24, 24))
    assert r.num_axes == 3 and r.axes == [0] * 16 + [1] * 24 + [2] * 24
    assert list(r._c.axis) == r.axes
    for i in (0, 1, 40, 63):
        f = 10000.0 ** (-i / 64)
        assert abs(r._c.turns[i] / 2.0 ** 64 * 2 * math.pi - f) < 1e-15
    # frequencies are taken modulo a turn: positions are whole
    r = qv.Rotary(dim=16, inv_freq=[-0.25 * math.pi, 2 * math.pi] + [0.0] * 6, axes=[1, 0] * 4, interleaved=True)
    # (pi in float64 is off by 2^-53 of itself, so these are by 2^11 of a turn's 2^64)
    assert abs(r._c.turns[0] - (2 ** 64 - 2 ** 61)) <= 2 ** 11
    assert min(r._c.turns[1], 2 ** 64 - r._c.turns[1]) <= 2 ** 11
    assert (r._c.num_pairs, r._c.num_axes, r._c.interleaved) == (8, 2, 1)
    # two axes that follow no pair are allowed to be last (a section of none)
    assert qv.Rotary(sections=(64, 0)).num_axes == 2


# ------------------------------------------------------------ advance
class _Lens(qv.BlockCache):
    """A cache's lengths alone, on the CPU."""

    def __init__(self, lens, max_context):
        self.torch, self.stream = torch, None
        self.cfg = qv.BlockConfig(len(lens), 8, 2, max_context)
        self._state = dict(lens=torch.tensor(lens, dtype=torch.int32))


def test_advance_by_chunks():
    c = _Lens([0, 5, -1, 98, 100, 101, -(1 << 31), 90], 100)
    cu = torch.tensor([0, 3, 3, 7, 12, 14, 16, 18, 30], dtype=torch.int32)
    c.advance(cu)
    assert c.lens.tolist() == [3, 5, -1, 100, 100, 101, -(1 << 31), 100]
    c = _Lens([0, 5, 7, 1], 100)
    c.advance(torch.tensor([0, 3, 6, 9, 9], dtype=torch.int32), torch.tensor([2, -4, 9, 1], dtype=torch.int32))
    assert c.lens.tolist() == [2, 5, 10, 1] and c.lens.dtype is torch.int32
    c.advance()
    assert c.lens.tolist() == [3, 6, 11, 2]


def test_a_cache_refuses_a_chunk_it_was_not_made_for():
    c = _Lens([0], 100)
    c.device = torch.device("cuda", 0)
    x = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="chunk_tokens"):
        c.attend_chunk(0, x, x, x, None, x)
    with pytest.raises(ValueError):
        c.append(0, x, x, None, positions=x)
    with pytest.raises(ValueError):
        c.append(0, x, x, None, rotary=qv.Rotary())
