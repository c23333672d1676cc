"""Rotary positions against float64.

Tolerance of an output: cos and sin are off by 2^-22 at most (the angle by 2^-33 turns, its
rounding to fp32 by 2^-24 of at most pi / 4, the series and its roundings by 2^-23), two fp32
products and their sum by 2^-23 of the pair's magnitudes, the result is rounded once to bf16
(2^-8 of itself): |error| <= 2^-8 |o| + 2^-21 (|x| + |y|).  Below 2^-126 the step of bf16 is
2^-133 whatever the value, of fp32 2^-149: half of one and a few of the others, 2^-134 +
2^-147, come on top."""
import fractions
import math

import pytest

pytestmark = pytest.mark.gpu
D = 128


def _bf16(*shape, seed=0, scale=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).bfloat16()


def _positions(T, axes, seed=0, lo=0, hi=131072):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randint(lo, hi, (T, axes), generator=g).to(torch.int32).cuda()


def _reference(x, positions, r, inverse=False):
    """(float64 result, |x| + |y| of every output's pair), on the CPU."""
    import torch
    x = x.double().cpu()
    positions = positions.double().cpu().view(x.shape[0], r.num_axes)
    n = r.dim // 2
    t = positions[:, r.axes] * torch.tensor(r.inv_freq, dtype=torch.float64)
    if float(positions.abs().max()) >= 2.0 ** 24:   # the float64 product would be off by too much
        pi = fractions.Fraction("3.14159265358979323846264338327950288419716939937510582097494")
        t = torch.tensor([[float(int(p) * fractions.Fraction(f) % (2 * pi)) for p, f in zip(row, r.inv_freq)]
                          for row in positions[:, r.axes].tolist()], dtype=torch.float64)
    t = (-t if inverse else t)[:, None]
    a = torch.arange(n) * 2 if r.interleaved else torch.arange(n)
    b = a + 1 if r.interleaved else a + n
    out, size = x.clone(), torch.zeros_like(x)
    out[..., a] = x[..., a] * t.cos() - x[..., b] * t.sin()
    out[..., b] = x[..., b] * t.cos() + x[..., a] * t.sin()
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def _check(got, x, positions, r, inverse=False):
    want, size = _reference(x, positions, r, inverse)
    err = (got.double().cpu() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + 2.0 ** -21 * size + 2.0 ** -134 + 2.0 ** -147).all()), err.max().item()
    if r.dim < D:
        assert (got[..., r.dim:] == x[..., r.dim:]).all()


CONFIGS = [
    dict(), dict(base=500000.0), dict(sections=(16, 24, 24)), dict(sections=(16, 16, 16, 16)), dict(interleaved=True),
    dict(dim=64), dict(dim=96, sections=(8, 20, 20)), dict(dim=16, interleaved=True), dict(dim=48, base=100.0),
    dict(axes=[0, 1, 2] * 21 + [0]), dict(axes=[1, 0] * 32, interleaved=True),
    dict(dim=112, interleaved=True, axes=[0, 1, 1, 0] * 14),
    dict(inv_freq=[0.3 * (-1) ** i / (i + 1) for i in range(64)]),
]


@pytest.mark.parametrize("kw", CONFIGS, ids=lambda k: "-".join(k) or "plain")
@pytest.mark.parametrize("T", [1, 31, 33, 500])
def test_rotate(kw, T):
    import paper_2608_05326_amd as qv
    r = qv.Rotary(**kw)
    q, k = _bf16(T, 5, D, seed=T), _bf16(T, 2, D, seed=T + 1)
    pos = _positions(T, r.num_axes, seed=T)
    qo, ko = qv.rotate(q, k, pos, r)
    _check(qo, q, pos, r)
    _check(ko, k, pos, r)
    qi, ki = qv.rotate(q, k, pos, r, inverse=True)
    _check(qi, q, pos, r, inverse=True)
    _check(ki, k, pos, r, inverse=True)


@pytest.mark.parametrize("hq,hk", [(1, 0), (1, 1), (7, 0), (8, 8), (9, 1), (64, 8), (28, 4), (130, 3)])
@pytest.mark.parametrize("T", [1, 4, 67])
def test_heads(hq, hk, T):
    import paper_2608_05326_amd as qv
    r = qv.Rotary()
    q, k = _bf16(T, hq, D, seed=hq), _bf16(T, hk, D, seed=hk) if hk else None
    pos = _positions(T, 1, seed=hq)[:, 0].contiguous()
    qo, ko = qv.rotate(q, k, pos, r)
    _check(qo, q, pos, r)
    if hk:
        _check(ko, k, pos, r)
    else:
        assert ko is None


@pytest.mark.parametrize("T,hq,hk", [(1500, 40, 3), (4200, 20, 3), (9001, 20, 3), (3000, 64, 8)])
def test_more_tokens_take_more_heads_a_workgroup(T, hq, hk):
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(sections=(16, 24, 24))
    q, k = _bf16(T, hq, D, seed=hq), _bf16(T, hk, D, seed=hk)
    pos = _positions(T, 3, seed=hq)
    qo, ko = qv.rotate(q, k, pos, r)
    rows = slice(T - 300, None)
    _check(qo[rows], q[rows], pos[rows], r)
    _check(ko[rows], k[rows], pos[rows], r)
    for x, o in ((q, qo), (k, ko)):       # every row: its own call, in pieces of few tokens, gives the same bits
        parts = [qv.rotate(x[i:i + 250], None, pos[i:i + 250], r)[0] for i in range(0, T, 250)]
        assert torch.equal(torch.cat(parts), o)


def test_positions_of_every_size():
    """The whole range of 32 bits, where an fp32 angle would be off by turns."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary()
    pos = torch.tensor([0, 1, -1, 2, 1 << 20, (1 << 24) + 1, -(1 << 24) - 1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2,
                        123456789, -987654321], dtype=torch.int32).cuda()
    q, k = _bf16(len(pos), 4, D, seed=1), _bf16(len(pos), 4, D, seed=2)
    qo, ko = qv.rotate(q, k, pos, r)
    _check(qo, q, pos, r)
    _check(ko, k, pos, r)
    assert torch.equal(qo[0], q[0])       # position 0 changes nothing


def test_quarter_turns_are_exact():
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(inv_freq=[math.pi / 2] * 64)
    x = _bf16(4, 1, D, seed=3)
    qo, _ = qv.rotate(x, None, torch.arange(4, dtype=torch.int32, device="cuda"), r)
    a, b = x[..., :64], x[..., 64:]
    for i, want in enumerate((torch.cat([a, b], -1), torch.cat([-b, a], -1), torch.cat([-a, -b], -1),
                              torch.cat([b, -a], -1))):
        assert (qo[i].float() - want[i].float()).abs().max() <= 2.0 ** -20 * 8


def test_strides_and_in_place():
    """Slices of a projection, [H, T, d] tensors, positions by axis, rotation in place."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(sections=(20, 22, 22))
    T, hq, hk = 77, 6, 2
    pos = _positions(3, T, seed=5).t()                      # [T, 3], strides (1, T)
    assert not pos.is_contiguous()
    buf = _bf16(T, hq + 2 * hk, D, seed=6)
    before = buf.clone()
    q, k = buf[:, :hq], buf[:, hq:hq + hk]
    qt = torch.empty(hq, T, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    kt = torch.full((T, 3 * hk, D), 7.0, dtype=torch.bfloat16, device="cuda")
    qv.rotate(q, k, pos, r, qt, kt[:, ::3])
    _check(qt, q, pos, r)
    _check(kt[:, ::3], k, pos, r)
    assert bool((kt[:, 1::3] == 7.0).all()) and torch.equal(buf, before)
    qo, ko = qv.rotate(q, k, pos, r, q, k)
    assert qo is q and ko is k and torch.equal(q, qt) and torch.equal(k, kt[:, ::3])
    assert torch.equal(buf[:, hq + hk:], before[:, hq + hk:])
    # back again: two roundings
    qv.rotate(q, k, pos, r, q, k, inverse=True)
    assert (q.float() - before[:, :hq].float()).abs().max() <= 2.0 ** -7 * before.abs().max().float() * 1.5
    one = _bf16(1, hq, D, seed=9)
    p1 = pos[:1]
    q1, _ = qv.rotate(one.expand(1, hq, D), None, p1, r)
    _check(q1, one, p1, r)


def test_values_that_are_not_finite_stay_in_their_pairs():
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary()
    x = _bf16(3, 2, D, seed=7)
    y = x.clone()
    y[1, 0, 5] = float("inf")
    y[2, 1, 100] = float("nan")
    pos = torch.tensor([3, 4, 5], dtype=torch.int32).cuda()
    a, _ = qv.rotate(x, None, pos, r)
    b, _ = qv.rotate(y, None, pos, r)
    touched = torch.zeros_like(x, dtype=torch.bool)
    touched[1, 0, [5, 69]] = True
    touched[2, 1, [36, 100]] = True
    assert torch.equal(a[~touched], b[~touched]) and not bool(b[touched].isfinite().any())


def test_sizes_of_values():
    """Tiny and huge values keep their bits (the products stay in the range of fp32)."""
    import paper_2608_05326_amd as qv
    r = qv.Rotary()
    pos = _positions(64, 1, seed=8)
    for scale in (2.0 ** -115, 2.0 ** -60, 2.0 ** 60, 2.0 ** 120):
        q = _bf16(64, 2, D, seed=9, scale=scale)
        qo, _ = qv.rotate(q, None, pos, r)
        _check(qo, q, pos, r)


def test_relative_positions():
    """Products of rotated queries and keys follow the difference of positions alone."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(sections=(16, 24, 24))
    T = 64
    q, k = _bf16(1, 1, D, seed=10).expand(T, 1, D).contiguous(), _bf16(1, 1, D, seed=11).expand(T, 1, D).contiguous()
    pos = _positions(T, 3, seed=12)
    shift = torch.tensor([5, -7, 11], dtype=torch.int32, device="cuda")
    a, _ = qv.rotate(q, None, pos, r)
    b, _ = qv.rotate(k, None, pos + shift, r)
    s = (a.double() * b.double()).sum(-1).flatten()
    # each rotated value is off by 2^-8 of itself at most: |q||k| 2 x 2^-8, and as much in the other
    bound = 4 * 2.0 ** -8 * (q[0].double().norm() * k[0].double().norm())
    assert (s - s[0]).abs().max() <= bound


def test_the_inverse_takes_gradients():
    """Against differences: f(x) = <g, rotate(x)> is linear, its gradient rotate(g, inverse)."""
    import paper_2608_05326_amd as qv
    r = qv.Rotary(sections=(16, 24, 24), interleaved=True)
    T = 9
    pos = _positions(T, 3, seed=13)
    g = _bf16(T, 2, D, seed=14)
    grad, _ = qv.rotate(g, None, pos, r, inverse=True)
    x, dx = _bf16(T, 2, D, seed=15), _bf16(T, 2, D, seed=16)
    fx = (g.double() * qv.rotate(x, None, pos, r)[0].double()).sum(-1)
    x2 = (x.double() + dx.double()).bfloat16()
    fx2 = (g.double() * qv.rotate(x2, None, pos, r)[0].double()).sum(-1)
    want = (grad.double() * (x2.double() - x.double())).sum(-1)
    # roundings of both function values and of the gradient: 2^-8 of sum |g| |x| each (a pair's
    # length at most sqrt 2 of its larger entry)
    bound = 2.0 ** -8 * 1.5 * g.double().norm(dim=-1) * (x.double().norm(dim=-1) + x2.double().norm(dim=-1) +
                                                        (x2 - x).double().norm(dim=-1))
    assert bool(((fx2 - fx - want).abs() <= bound).all())


def test_refusals_and_streams():
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(sections=(16, 24, 24))
    q, k = _bf16(10, 4, D), _bf16(10, 2, D)
    pos = _positions(10, 3)
    for bad in (pos[:9], pos[:, :2], pos.long(), pos.cpu(), pos[:, 0]):
        with pytest.raises(ValueError):
            qv.rotate(q, k, bad, r)
    with pytest.raises(ValueError):
        qv.rotate(q, k[:9], pos, r)
    with pytest.raises(ValueError):
        qv.rotate(q.float(), k, pos, r)
    with pytest.raises(ValueError):
        qv.rotate(q, None, pos, r, k_out=k)
    with pytest.raises(qv.QEvictError):
        qv.rotate(q[..., :64], k[..., :64], pos, r)
    with pytest.raises(qv.QEvictError):
        qv.rotate(q, k, pos, r, q_out=torch.empty(1, 4, D, dtype=torch.bfloat16, device="cuda").expand(10, 4, D))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want, _ = qv.rotate(q, k, pos, r)
    torch.cuda.synchronize()
    got, _ = qv.rotate(q, k, pos, r, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    e, f = qv.rotate(q[:0], k[:0], pos[:0], r)
    assert e.shape == (0, 4, D) and f.shape == (0, 2, D)


def test_captured():
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary()
    q, k, pos = _bf16(40, 4, D, seed=1), _bf16(40, 2, D, seed=2), _positions(40, 1, seed=3)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        qv.rotate(q, k, pos, r, qo, ko)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        qv.rotate(q, k, pos, r, qo, ko)
    for i in range(4):
        pos.copy_(_positions(40, 1, seed=20 + i))
        g.replay()
        torch.cuda.synchronize()
        want, wk = qv.rotate(q, k, pos, r)
        assert torch.equal(qo, want) and torch.equal(ko, wk)


def test_rows_past_2_to_the_31():
    """Rows further than 2^31 elements from the first."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary()
    T, st = 600, 1 << 22
    buf = torch.empty((T - 1) * st + 2 * D, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((T, 2, D), (st, D, 1))
    x = _bf16(T, 2, D, seed=4)
    q.copy_(x)
    pos = _positions(T, 1, seed=5)
    qo, _ = qv.rotate(q, None, pos, r, q)
    _check(qo, x, pos, r)
