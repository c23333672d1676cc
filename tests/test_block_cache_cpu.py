"""Host-side refusals of the packed-prompt and block-cache calls: every one is decided
before anything touches a device, so they are checked here without a GPU (the pointers are
never followed)."""
import ctypes

import pytest

import paper_2608_05326_amd as qv
from paper_2608_05326_amd import qevict as m

P = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 8)


def _prompt(q=P, k=P, v=P, cu=P, out=P, **kw):
    c = m._PromptConfig(qv.qevict.ABI_VERSION, 2, 100, 8, 2, 128, 0.0, 1024, 128, 256, 128, 256, 128, 1024, 128)
    for n, x in kw.items():
        setattr(c, n, x)
    return qv.load_library().qevict_prompt_attend(ctypes.byref(c), q, k, v, cu, out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=3), m.ERR_UNSUPPORTED),
    (dict(head_dim=64), m.ERR_UNSUPPORTED),
    (dict(num_q_heads=0), m.ERR_INVALID_ARG),
    (dict(num_q_heads=9), m.ERR_INVALID_ARG),
    (dict(num_kv_heads=-1), m.ERR_INVALID_ARG),
    (dict(num_seqs=0), m.ERR_INVALID_ARG),
    (dict(total_tokens=-1), m.ERR_INVALID_ARG),
    (dict(softmax_scale=-1.0), m.ERR_INVALID_ARG),
    (dict(softmax_scale=float("nan")), m.ERR_INVALID_ARG),
    (dict(softmax_scale=float("inf")), m.ERR_INVALID_ARG),
    (dict(q=None), m.ERR_INVALID_ARG),
    (dict(k=ODD), m.ERR_INVALID_ARG),
    (dict(cu=None), m.ERR_INVALID_ARG),
    (dict(cu=ctypes.c_void_p(2)), m.ERR_INVALID_ARG),
    (dict(out=ODD), m.ERR_INVALID_ARG),
    (dict(v_token_stride=-256), m.ERR_INVALID_ARG),
    (dict(k_head_stride=132), m.ERR_INVALID_ARG),
    (dict(q_token_stride=1 << 60), m.ERR_INVALID_ARG),
    (dict(out_token_stride=512), m.ERR_INVALID_ARG),        # rows overlap
    (dict(out_head_stride=0), m.ERR_INVALID_ARG),
    (dict(total_tokens=1 << 28, out_token_stride=1024), m.ERR_UNSUPPORTED),
    (dict(num_seqs=1 << 30), m.ERR_UNSUPPORTED),
    (dict(k_token_stride=1 << 23), m.ERR_UNSUPPORTED),
    (dict(v_token_stride=1 << 24), m.ERR_UNSUPPORTED),
])
def test_prompt_attend_refuses(kw, status):
    assert _prompt(**kw) == status
    assert qv.load_library().qevict_last_error()


def test_nothing_to_do_is_ok():
    assert _prompt(total_tokens=0, q=None, k=None, v=None, out=None) == m.OK


def _block(call, cfg=None, layer=None, **kw):
    lib = qv.load_library()
    c = m._BlockConfig(qv.qevict.ABI_VERSION, 2, 8, 2, 128, 1000, 40, 0.0)
    for n, x in (cfg or {}).items():
        setattr(c, n, x)
    p = m._BlockLayer(*[1 << 20] * 8)
    for n, x in (layer or {}).items():
        setattr(p, n, x)
    if call == "attend":
        a = dict(q=P, k=P, v=P, out=P, ws=P, size=1 << 40)
        a.update(kw)
        return lib.qevict_block_attend(ctypes.byref(c), ctypes.byref(p), a["q"], a["k"], a["v"], a["out"],
                                       a["ws"], a["size"], None)
    a = dict(k=P, k_st=256, k_sh=128, v=P, v_st=256, v_sh=128, cu=P, total=100)
    a.update(kw)
    fn = lib.qevict_block_store if call == "store" else lib.qevict_block_fetch
    return fn(ctypes.byref(c), ctypes.byref(p), a["k"], a["k_st"], a["k_sh"], a["v"], a["v_st"], a["v_sh"],
              a["cu"], a["total"], None)


@pytest.mark.parametrize("call", ["store", "fetch", "attend"])
@pytest.mark.parametrize("cfg,layer,status", [
    (dict(abi_version=5), {}, m.ERR_UNSUPPORTED),
    (dict(head_dim=96), {}, m.ERR_UNSUPPORTED),
    (dict(num_q_heads=34), {}, m.ERR_UNSUPPORTED),          # 17 heads per KV head
    (dict(num_q_heads=7), {}, m.ERR_INVALID_ARG),
    (dict(batch=0), {}, m.ERR_INVALID_ARG),
    (dict(max_context=0), {}, m.ERR_INVALID_ARG),
    (dict(max_context=(1 << 30) + 1), {}, m.ERR_UNSUPPORTED),
    (dict(num_pages=-1), {}, m.ERR_INVALID_ARG),
    (dict(batch=1 << 24), {}, m.ERR_UNSUPPORTED),
    (dict(softmax_scale=-0.5), {}, m.ERR_INVALID_ARG),
    ({}, dict(k_codes=0), m.ERR_INVALID_ARG),
    ({}, dict(v_codes=(1 << 20) + 8), m.ERR_INVALID_ARG),
    ({}, dict(v_scale=0), m.ERR_INVALID_ARG),
    ({}, dict(k_tail=0), m.ERR_INVALID_ARG),
    ({}, dict(v_tail=(1 << 20) + 2), m.ERR_INVALID_ARG),
    ({}, dict(table=0), m.ERR_INVALID_ARG),
    ({}, dict(lens=(1 << 20) + 1), m.ERR_INVALID_ARG),
])
def test_block_calls_refuse(call, cfg, layer, status):
    assert _block(call, cfg, layer) == status


@pytest.mark.parametrize("call", ["store", "fetch"])
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), m.ERR_INVALID_ARG),
    (dict(v=ODD), m.ERR_INVALID_ARG),
    (dict(k_st=-256), m.ERR_INVALID_ARG),
    (dict(v_sh=4), m.ERR_INVALID_ARG),
    (dict(cu=None), m.ERR_INVALID_ARG),
    (dict(total=-1), m.ERR_INVALID_ARG),
])
def test_packed_calls_refuse(call, kw, status):
    assert _block(call, **kw) == status


def test_fetch_refuses_rows_that_overlap_and_attend_its_tensors():
    assert _block("fetch", k_st=128) == m.ERR_INVALID_ARG
    assert _block("fetch", v_sh=0) == m.ERR_INVALID_ARG
    for kw in (dict(q=None), dict(k=ODD), dict(v=ODD), dict(out=ctypes.c_void_p((1 << 20) + 2))):
        assert _block("attend", **kw) == m.ERR_INVALID_ARG
    for kw in (dict(ws=None), dict(ws=ODD), dict(size=0), dict(size=1000)):
        assert _block("attend", **kw) == m.ERR_WORKSPACE
    assert _block("store", total=0, k=None, v=None, cu=None) == m.OK


def test_workspace_size():
    lib = qv.load_library()
    c = m._BlockConfig(qv.qevict.ABI_VERSION, 2, 8, 2, 128, 1000, 40, 0.0)
    n = ctypes.c_size_t()
    assert lib.qevict_block_workspace_size(ctypes.byref(c), ctypes.byref(n)) == m.OK
    # a partial row of 128 values, maximum and sum per head of a (part or pair): 4 heads a pair
    assert n.value % (4 * 130 * 4) == 0 and n.value // (4 * 130 * 4) > 2 * 2
    assert _block("attend", size=n.value - 1) == m.ERR_WORKSPACE
    c.batch = 0
    assert lib.qevict_block_workspace_size(ctypes.byref(c), ctypes.byref(n)) == m.ERR_INVALID_ARG
    assert lib.qevict_block_workspace_size(None, ctypes.byref(n)) == m.ERR_INVALID_ARG


def test_a_block_cache_needs_a_gpu():
    with pytest.raises(ValueError):
        qv.BlockCache(qv.BlockConfig(1, 8, 2, 100), device="cpu")
