"""Causal attention of packed prompts (prompt_attend) against float64 on the CPU.

Tolerance, per output element: the kernel rounds each probability to bf16 once (half a
step, 2^-8 relative) and the output once, so with A = sum_j p_j |v_j| the result is off by
at most 2^-8 (A + |o|); logits are fp32 sums of exact products (128 terms: |error| below
2^-24 x 128 x sum|q k| scale, under 2^-12 for these inputs), which enters twice (numerator
and sum): 2^-11 A more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
D = 128


def _inputs(lens, hq, hkv, seed=0, layout="separate", extra=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    T = sum(lens) + extra

    def rnd(*s):
        return torch.randn(*s, generator=g).bfloat16()
    if layout == "fused":
        x = rnd(T, hq + 2 * hkv, D).cuda()
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    elif layout == "heads_first":
        q, k, v = (rnd(h, T, D).cuda().transpose(0, 1) for h in (hq, hkv, hkv))
    else:
        q, k, v = (rnd(T, h, D).cuda() for h in (hq, hkv, hkv))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    return q, k, v, cu


def _reference(q, k, v, lens, scale=D ** -0.5):
    """float64 output and sum_j p_j |v_j|; masked keys take no part whatever they hold."""
    import torch
    q, k, v = (x.double().cpu() for x in (q, k, v))
    o, A = torch.zeros_like(q), torch.zeros_like(q)
    G = q.shape[1] // k.shape[1]
    a = 0
    for t in lens:
        mask = torch.ones(t, t, dtype=torch.bool).tril()
        for h in range(q.shape[1]):
            kk, vv = k[a:a + t, h // G], v[a:a + t, h // G]
            s = (q[a:a + t, h] @ kk.T) * scale
            p = torch.softmax(s.masked_fill(~mask, -torch.inf), dim=1)
            fin = torch.where(torch.isfinite(vv), vv, 0.0)
            o[a:a + t, h] = p @ fin
            A[a:a + t, h] = p @ fin.abs()
            for j in torch.nonzero(~torch.isfinite(vv).all(1))[:, 0].tolist():
                bad = torch.where(torch.isfinite(vv[j]), 0.0, vv[j])
                o[a + j:a + t, h] += bad
        a += t
    return o, A


def _check(out, o, A, what=""):
    import torch
    out = out.double().cpu()
    fin = torch.isfinite(o)
    assert bool((torch.isfinite(out) == fin).all()), what
    same = (out == o) | (torch.isnan(out) & torch.isnan(o))
    assert bool(same[~fin].all()), what
    tol = (2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A)[fin]
    err = (out - o).abs()[fin]
    assert bool((err <= tol).all()), (what, (err / tol).max().item())


LENS = [[1], [2], [63], [64], [65], [127, 1, 129], [0, 5, 0, 0, 200, 0], [31, 33, 300], [777],
        list(range(1, 80)), [1500]]


@pytest.mark.parametrize("lens", LENS, ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (8, 2), (7, 1), (12, 4)])
def test_packed_prompts(lens, hq, hkv):
    import torch
    import paper_2608_05326_amd as qv
    q, k, v, cu = _inputs(lens, hq, hkv, seed=len(lens) + hq)
    out = qv.prompt_attend(q, k, v, cu)
    torch.cuda.synchronize()
    _check(out, *_reference(q, k, v, lens))


@pytest.mark.parametrize("hq,hkv", [(16, 1), (20, 1), (64, 8)])
def test_wide_groups(hq, hkv):
    import paper_2608_05326_amd as qv
    lens = [3, 150, 17]
    q, k, v, cu = _inputs(lens, hq, hkv, seed=5)
    _check(qv.prompt_attend(q, k, v, cu), *_reference(q, k, v, lens))


def test_many_prompts():
    """Thousands of short prompts, empty ones among them, rows before the first."""
    import torch
    import paper_2608_05326_amd as qv
    lens = np.random.default_rng(0).integers(0, 12, 5000).tolist()
    q, k, v, cu = _inputs(lens, 2, 1, seed=1, extra=40)
    out = torch.full_like(q, 7.0)
    qv.prompt_attend(q, k, v, cu, out)
    n = sum(lens)
    _check(out[:n], *_reference(q[:n], k[:n], v[:n], lens))
    assert bool((out[n:] == 7.0).all())
    out2 = torch.full_like(q, 7.0)
    qv.prompt_attend(q, k, v, cu[70:].contiguous(), out2)
    a = int(cu[70])
    assert bool((out2[:a] == 7.0).all()) and torch.equal(out2[a:], out[a:])


@pytest.mark.parametrize("layout", ["fused", "heads_first"])
def test_strides(layout):
    import torch
    import paper_2608_05326_amd as qv
    lens = [130, 7, 65]
    q, k, v, cu = _inputs(lens, 8, 2, seed=9, layout=layout)
    out = torch.empty(8, sum(lens), D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    qv.prompt_attend(q, k, v, cu, out)
    _check(out, *_reference(q, k, v, lens))


def test_shared_head_and_scale():
    """A KV tensor expanded over heads (stride 0) and a softmax scale of the caller's."""
    import paper_2608_05326_amd as qv
    lens = [90, 200]
    q, k, v, cu = _inputs(lens, 4, 1, seed=11)
    k2, v2 = k.expand(-1, 2, -1), v.expand(-1, 2, -1)
    _check(qv.prompt_attend(q, k2, v2, cu, softmax_scale=0.25), *_reference(q, k2, v2, lens, 0.25))


def test_rows_outside_the_prompts_stay():
    import torch
    import paper_2608_05326_amd as qv
    lens = [100, 29]
    q, k, v, cu = _inputs(lens, 8, 4, seed=2, extra=75)
    for x in (k, v):
        x[sum(lens):] = float("nan")
    out = torch.full_like(q, 7.0)
    qv.prompt_attend(q, k, v, cu, out)
    n = sum(lens)
    _check(out[:n], *_reference(q[:n], k[:n], v[:n], lens))
    assert bool((out[n:] == 7.0).all())
    # a first prompt that starts behind row 0
    cu2 = cu[1:].contiguous()
    out = torch.full_like(q, 7.0)
    qv.prompt_attend(q, k, v, cu2, out)
    _check(out[100:n], *_reference(q[100:n], k[100:n], v[100:n], [29]))
    assert bool((out[:100] == 7.0).all()) and bool((out[n:] == 7.0).all())


def test_bounds_outside_the_rows_are_clamped():
    import torch
    import paper_2608_05326_amd as qv
    q, k, v, cu = _inputs([100], 4, 4, seed=3)
    out = torch.full_like(q, 7.0)
    bad = torch.tensor([-5, 60, 40, 1 << 30], dtype=torch.int32, device="cuda")   # [0,60), none, [40,100)
    qv.prompt_attend(q[:60], k[:60], v[:60], bad[:2].contiguous(), out[:60])
    _check(out[:60], *_reference(q[:60], k[:60], v[:60], [60]))
    qv.prompt_attend(q, k, v, bad[2:].contiguous(), out)
    _check(out[40:], *_reference(q[40:], k[40:], v[40:], [60]))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 5, 63, 64, 100, 129])
def test_masked_values_that_are_not_finite(at, bad):
    """Value, key and query entries that are not finite reach the rows that see them only."""
    import paper_2608_05326_amd as qv
    lens = [130, 40]
    q, k, v, cu = _inputs(lens, 8, 2, seed=4)
    v[at, 0, 3] = bad
    v[at, 1, 127] = bad
    out = qv.prompt_attend(q, k, v, cu)
    o, A = _reference(q, k, v, lens)
    _check(out, o, A, "value")
    q, k, v, cu = _inputs(lens, 8, 2, seed=6)
    want, A = _reference(q, k, v, lens)
    k[at, 1, 9] = bad
    out = qv.prompt_attend(q, k, v, cu)
    _check(out[:, :4], want[:, :4], A[:, :4], "other KV head")
    _check(out[:at, 4:], want[:at, 4:], A[:at, 4:], "rows before the key")
    _check(out[130:], want[130:], A[130:], "other prompt")
    q, k, v, cu = _inputs(lens, 8, 2, seed=6)
    q[at, 3, 9] = bad
    out = qv.prompt_attend(q, k, v, cu).clone()
    assert bool(out[at, 3].isnan().all())
    out[at, 3], want[at, 3], A[at, 3] = 0, 0, 0
    _check(out, want, A, "query")


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 31, 32, 127, 128, 200, 299])
def test_masked_values_of_a_lone_prompt(at, bad):
    """The same where a few long rows are shared by four waves each (one prompt, few heads)."""
    import paper_2608_05326_amd as qv
    q, k, v, cu = _inputs([300], 2, 1, seed=15)
    v[at, 0, 5] = bad
    _check(qv.prompt_attend(q, k, v, cu), *_reference(q, k, v, [300]))
    q, k, v, cu = _inputs([300], 2, 1, seed=16)
    want, A = _reference(q, k, v, [300])
    k[at, 0, 9] = bad
    out = qv.prompt_attend(q, k, v, cu)
    _check(out[:at], want[:at], A[:at], "rows before the key")


def test_large_and_shifted_logits():
    """Logits in the hundreds (one key takes a row), rising and falling along the prompt."""
    import torch
    import paper_2608_05326_amd as qv
    lens = [500]
    q, k, v, cu = _inputs(lens, 4, 2, seed=8)
    ramp = torch.linspace(-30, 30, 500, device="cuda")[:, None, None]
    for r in (ramp, -ramp):
        k2 = (k.float() + r).bfloat16()
        out = qv.prompt_attend(q, k2, v, cu)
        o, A = _reference(q, k2, v, lens)
        # logit error: 2^-24 x 128 terms x sum|q k| scale (up to 128 x 4 x 34 / 11.3 = 1540)
        d = 2.0 ** -24 * 128 * 1540
        err = (out.double().cpu() - o).abs()
        assert bool((err <= 2.0 ** -8 * (A + o.abs()) + 4 * d * A).all())


def test_long_prompt_rows():
    """A 9000-token prompt: sampled rows against float64."""
    import torch
    import paper_2608_05326_amd as qv
    T = 9000
    q, k, v, cu = _inputs([T], 8, 2, seed=12, layout="fused")
    out = qv.prompt_attend(q, k, v, cu).double().cpu()
    q, k, v = (x.double().cpu() for x in (q, k, v))
    for i in list(range(0, T, 611)) + [T - 1]:
        for h in (0, 3, 7):
            p = torch.softmax(k[:i + 1, h // 4] @ q[i, h] * D ** -0.5, 0)
            o, A = p @ v[:i + 1, h // 4], p @ v[:i + 1, h // 4].abs()
            assert bool(((out[i, h] - o).abs() <= 2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A).all()), (i, h)


def test_repeats_bitwise_and_on_another_stream():
    import torch
    import paper_2608_05326_amd as qv
    lens = [700, 3, 1500]
    q, k, v, cu = _inputs(lens, 8, 2, seed=13)
    a = qv.prompt_attend(q, k, v, cu)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    b = torch.empty_like(a)
    qv.prompt_attend(q, k, v, cu, b, stream=st)
    st.synchronize()
    with torch.cuda.stream(st):
        c = qv.prompt_attend(q, k, v, cu)
    st.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def test_captured_with_lengths_read_at_replay():
    import torch
    import paper_2608_05326_amd as qv
    q, k, v, cu = _inputs([100, 300], 8, 2, seed=14)
    out = torch.zeros_like(q)
    qv.prompt_attend(q, k, v, cu, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qv.prompt_attend(q, k, v, cu, out)
    for lens in ([100, 300], [399, 1], [0, 400], [250, 150]):
        cu.copy_(torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32))
        out.zero_()
        graph.replay()
        want = qv.prompt_attend(q, k, v, cu)
        torch.cuda.synchronize()
        assert torch.equal(out, want), lens
        _check(out, *_reference(q, k, v, lens))


def test_refusals():
    import torch
    import paper_2608_05326_amd as qv
    q, k, v, cu = _inputs([40], 8, 2)
    out = torch.full_like(q, 7.0)
    wide = torch.zeros(40, 8, 2 * D, dtype=torch.bfloat16, device="cuda")
    for bad in [dict(q=q.float()), dict(k=k.cpu()), dict(v=v[:39]), dict(k=k[:, :1]), dict(out=out[:, :4]),
                dict(q=q[0]), dict(q=wide[:, :, ::2]), dict(cu=cu.long()), dict(cu=cu.cpu()),
                dict(q=q[..., :64], k=k[..., :64], v=v[..., :64], out=out[..., :64])]:
        a = dict(q=q, k=k, v=v, cu=cu, out=out)
        a.update(bad)
        with pytest.raises((ValueError, qv.QEvictError)):
            qv.prompt_attend(a["q"], a["k"], a["v"], a["cu"], a["out"])
    flat = torch.zeros(40 * 8 * D + 8, dtype=torch.bfloat16, device="cuda")
    for t, st in ((flat[1:], (8 * D, D, 1)), (flat, (8 * D + 4, D, 1)), (flat, (8 * D, D - 4, 1))):
        with pytest.raises(qv.QEvictError) as e:
            qv.prompt_attend(t.as_strided((40, 8, D), st) if st[0] == 8 * D else t.as_strided((39, 8, D), st),
                             *( (k, v, cu, out) if st[0] == 8 * D else (k[:39], v[:39], cu, out[:39])))
        assert e.value.status == qv.ERR_INVALID_ARG
    with pytest.raises(qv.QEvictError) as e:   # rows of out that overlap
        qv.prompt_attend(q, k, v, cu, out[:, :1].expand(-1, 8, -1))
    assert e.value.status == qv.ERR_INVALID_ARG
    with pytest.raises(qv.QEvictError) as e:   # three query heads on two KV heads
        qv.prompt_attend(q[:, :3], k, v, cu, out[:, :3])
    assert e.value.status == qv.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    empty = torch.zeros(0, 8, D, dtype=torch.bfloat16, device="cuda")
    assert qv.prompt_attend(empty, empty[:, :2], empty[:, :2], cu).shape == (0, 8, D)
