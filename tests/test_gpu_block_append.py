"""New tokens behind the tokens of a block cache: codes, scales and open blocks are decided
exactly, so everything is compared for equality (rotated keys with what qv.rotate gives)."""
import numpy as np
import pytest

from test_gpu_block_cache import D, N, _bf16, _check_closed, _cu, _make

pytestmark = pytest.mark.gpu


def _bits(x):
    import torch
    return x.view(torch.int16)


def _append(bc, held, lens, k, v, layer=0, kept=None, **kw):
    """One append at the given lengths, checked: what closes against exact arithmetic, the open
    blocks, and that nothing else is written.  k, v: [T, H_kv, d]; `kept` the keys that the
    cache is to hold (default k)."""
    import torch
    c = bc.cfg
    kept = k if kept is None else kept
    state = {n: getattr(bc, n).clone() for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")}
    counts = kw.get("counts")
    cu = np.concatenate([[0], np.cumsum(lens)])
    bc.append(layer, k, v, _cu(lens), **kw)
    torch.cuda.synchronize()
    written = set()
    for s, a in enumerate(held):
        n = 0 if a < 0 or a >= c.max_context else min(lens[s], c.max_context - a)
        if counts is not None:
            n = max(0, min(n, int(counts[s])))
        rows = []
        for x, tail in ((kept, "k_tail"), (v, "v_tail")):
            new = x[int(cu[s]):int(cu[s]) + n].transpose(0, 1)
            rows.append(torch.cat([state[tail][layer, s, :, :max(a, 0) % N], new], 1) if n else new)
        first = max(a, 0) // N
        done = (max(a, 0) % N + n) // N if n else 0
        for b in range(done):
            page = int(bc.table[s, first + b])
            if 0 <= page < bc.num_pages:
                written.add(page)
            _check_closed(bc, layer, s, first + b, *[x[:, b * N:(b + 1) * N] for x in rows])
        for x, tail in zip(rows, ("k_tail", "v_tail")):
            want = state[tail][layer, s].clone()
            if n:
                want[:, :x.shape[1] - done * N] = x[:, done * N:]
            assert torch.equal(_bits(getattr(bc, tail)[layer, s]), _bits(want)), (s, tail)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        keep = torch.ones(bc.num_pages, dtype=torch.bool)
        keep[list(written)] = False
        x, y = getattr(bc, name)[layer].cpu()[keep], state[name][layer].cpu()[keep]
        if x.dtype is not torch.int8:
            x, y = x.view(torch.int32), y.view(torch.int32)
        assert torch.equal(x, y), name
    return written


def _fresh(held, hkv, extra, seed=0, fill=0.0, **kw):
    """A cache whose places hold `held` tokens, with room for `extra` more each."""
    bc, _, _ = _make(held, 2 * hkv, hkv, max_context=max(max(held), 1) + extra, seed=seed, fill=fill, **kw)
    return bc


def _rows(T, hkv, seed):
    return [_bf16(T, hkv, D, seed=seed + i).cuda() for i in (0, 1)]


CASES = [
    ([0], [1]), ([0], [63]), ([0], [64]), ([0], [65]), ([0], [200]), ([63], [1]), ([63], [2]), ([64], [64]),
    ([1], [62]), ([1], [63]), ([1], [64]), ([1], [127]), ([1], [128]), ([40], [300]),
    ([10, 0, -1, 64, 100, 127], [5, 0, 9, 63, 28, 130]), ([3] * 70, [61] * 70), ([700], [1000]),
]


@pytest.mark.parametrize("held,lens", CASES, ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("hkv", [1, 3])
def test_append(held, lens, hkv):
    bc = _fresh(held, hkv, 1100, seed=len(lens) + sum(lens))
    _append(bc, held, lens, *_rows(sum(lens), hkv, seed=5))


@pytest.mark.parametrize("held,lens", CASES[5:], ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("kw", [dict(), dict(sections=(16, 24, 24)), dict(interleaved=True), dict(dim=96),
                                dict(dim=48, interleaved=True, sections=(12, 12))],
                         ids=lambda k: "-".join(k) or "plain")
def test_append_rotated(held, lens, kw):
    """The keys that qv.rotate gives, bit for bit, through every block end."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(**kw)
    T, hkv = sum(lens), 2
    bc = _fresh(held, hkv, 1100, seed=T)
    k, v = _rows(T, hkv, seed=6)
    g = torch.Generator().manual_seed(T)
    pos = torch.randint(0, 100000, (r.num_axes, T), generator=g).to(torch.int32).cuda().t()
    kept, _ = qv.rotate(k, None, pos, r)
    before = k.clone()
    _append(bc, held, lens, k, v, kept=kept, rotary=r, positions=pos)
    assert torch.equal(k, before)


@pytest.mark.parametrize("hkv,places", [(8, 40), (3, 115)])
@pytest.mark.parametrize("kw", [dict(), dict(dim=80, interleaved=True)], ids=lambda k: "-".join(k) or "plain")
def test_append_rotated_many(hkv, places, kw):
    """Calls large enough that a workgroup takes several heads, an odd number of them too."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(**kw)
    held = [(0, 3, 63, 64, 37)[s % 5] for s in range(places)]
    lens = [(130, 125, 1, 64, 190)[s % 5] for s in range(places)]
    bc = _fresh(held, hkv, 260, seed=places)
    k, v = _rows(sum(lens), hkv, seed=7)
    pos = torch.arange(sum(lens), dtype=torch.int32).cuda() * 3
    kept, _ = qv.rotate(k, None, pos, r)
    _append(bc, held, lens, k, v, kept=kept, rotary=r, positions=pos)


def test_pieces_give_what_a_store_gives():
    """A prompt appended in pieces of any size is the prompt stored at once, and rotated too."""
    import paper_2608_05326_amd as qv
    import torch
    r = qv.Rotary(base=500000.0)
    total, hkv = [1000, 64, 777, 130], 2
    a, k, v = _make(total, 4, hkv, seed=3)
    b = _fresh([0] * 4, hkv, max(total) + 70, seed=4)
    c = _fresh([0] * 4, hkv, max(total) + 70, seed=5)
    cu = np.concatenate([[0], np.cumsum(total)])
    pos = torch.cat([torch.arange(t) for t in total]).to(torch.int32).cuda()
    rng = np.random.default_rng(9)
    at = [0] * 4
    while any(x < t for x, t in zip(at, total)):
        n = [min(t - x, int(rng.integers(0, 150))) for x, t in zip(at, total)]
        rows = torch.cat([torch.arange(cu[s] + at[s], cu[s] + at[s] + n[s]) for s in range(4)]).long().cuda()
        for x, kw in ((b, {}), (c, dict(rotary=r, positions=pos[rows]))):
            x.append(0, k[rows], v[rows], _cu(n), **kw)
            x.advance(_cu(n))
        at = [x + y for x, y in zip(at, n)]
    assert b.lens.tolist() == total and c.lens.tolist() == total
    kr, _ = qv.rotate(k, None, pos, r)
    d = _fresh([0] * 4, hkv, max(total) + 70, seed=6)
    d.store(0, kr, v, _cu(total))
    d.lens = torch.tensor(total, dtype=torch.int32)
    out = []
    for x in (a, b, c, d):
        ko, vo = torch.zeros_like(k), torch.zeros_like(v)
        x.fetch(0, ko, vo, _cu(total))
        out.append((ko, vo))
    for x, y in ((0, 1), (3, 2)):
        assert torch.equal(out[x][0], out[y][0]) and torch.equal(out[x][1], out[y][1])
    assert not torch.equal(out[0][0], out[3][0])


def test_counts():
    import torch
    held, lens = [60, 5, 0, 100, 64, 1], [8, 8, 130, 8, 5, 3]
    bc = _fresh(held, 2, 300, seed=1)
    for counts in ([8, 0, 65, 28, -3, 2], [0] * 6, [1 << 30, 1, 1, -(1 << 31), 5, 3]):
        _append(bc, held, lens, *_rows(sum(lens), 2, seed=7),
                counts=torch.tensor(counts, dtype=torch.int32).cuda())


def test_room_and_places_without_a_sequence():
    import torch
    held = [100, -1, 130, 129, 66]
    bc, _, _ = _make([100, -1, 130, 129, 66], 4, 2, max_context=130, seed=5, fill=0.0)
    lens = [40, 7, 3, 2, 64]
    _append(bc, held, lens, *_rows(sum(lens), 2, seed=8))
    bc.lens = torch.tensor([-7, 1 << 30, -(1 << 31), 131, 2 ** 31 - 1], dtype=torch.int32)
    _append(bc, [-7, 1 << 30, -1, 131, 2 ** 31 - 1], lens, *_rows(sum(lens), 2, seed=9))


@pytest.mark.parametrize("drop", [-1, 1 << 30, -(1 << 31)])
def test_blocks_without_a_page(drop):
    """Their tokens are not stored; the open block behind them is."""
    held, lens = [30, 64, 10], [200, 70, 55]
    bc = _fresh(held, 2, 300, seed=2)
    bc.table[0, 0] = bc.table[0, 2] = bc.table[1, 1] = bc.table[2, 0] = drop
    written = _append(bc, held, lens, *_rows(sum(lens), 2, seed=10))
    assert len(written) == 1


def test_strided_rows_and_rows_outside_the_places():
    """Slices of a projection and [H, T, d] tensors; rows before, between and behind are not read
    (NaN), bounds outside the rows are clamped."""
    import paper_2608_05326_amd as qv
    import torch
    held, lens, hkv = [10, 64, 3], [60, 64, 100], 2
    T = 300
    buf = torch.full((T, 8 + 2 * hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    k, v = _rows(sum(lens), hkv, seed=11)
    cu = torch.tensor([20, 80, 144, 244], dtype=torch.int32).cuda()
    buf[20:244, 8:8 + hkv], buf[20:244, 8 + hkv:] = k, v
    a, b = _fresh(held, hkv, 300, seed=3), _fresh(held, hkv, 300, seed=3)
    a.append(0, k, v, _cu(lens))
    b.append(0, buf[:, 8:8 + hkv], buf[:, 8 + hkv:], cu)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    b = _fresh(held, hkv, 300, seed=3)
    kt = k.transpose(0, 1).contiguous().transpose(0, 1)
    b.append(0, kt, v, torch.tensor([-5, 60, 124, 1 << 30], dtype=torch.int32).cuda())
    assert torch.equal(a.k_codes, b.k_codes) and torch.equal(a.v_tail, b.v_tail)
    # positions by row, not by place
    r = qv.Rotary()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 3
    kr, _ = qv.rotate(k, None, pos[20:244].contiguous(), r)
    a, b = _fresh(held, hkv, 300, seed=3), _fresh(held, hkv, 300, seed=3)
    a.append(0, kr, v, _cu(lens))
    b.append(0, buf[:, 8:8 + hkv], buf[:, 8 + hkv:], cu, r, pos)
    assert torch.equal(a.k_codes, b.k_codes) and torch.equal(a.k_tail, b.k_tail)


def test_values_that_are_not_finite():
    import torch
    held, lens = [30, 30, 0], [40, 40, 128]
    bc = _fresh(held, 2, 300, seed=4)
    k, v = _rows(sum(lens), 2, seed=12)
    k[3, 1, 7] = float("inf")
    v[45, 0, 99] = float("nan")
    k[80 + 100, 0, 0] = float("-inf")
    bc.k_tail[0, 1, 1, 4, 4] = float("nan")
    _append(bc, held, lens, k, v)


def test_many_places():
    rng = np.random.default_rng(13)
    held = rng.integers(-1, 130, 300).tolist()
    lens = rng.integers(0, 6, 300)
    lens[[5, 63, 64, 130, 299]] = [300, 64, 1, 127, 200]
    bc = _fresh(held, 1, 320, seed=14)
    _append(bc, held, lens.tolist(), *_rows(int(lens.sum()), 1, seed=15))


def test_layers_and_captured_appends():
    """Two layers of one cache, captured once and replayed while the lengths move."""
    import paper_2608_05326_amd as qv
    import torch
    held, lens, hkv = [50, 0, 120], [9, 3, 17], 2
    bc, k0, _ = _make(held, 4, hkv, max_context=400, layers=2, seed=16, fill=0.0)
    ref, _, _ = _make(held, 4, hkv, max_context=400, layers=2, seed=16, fill=0.0)
    r = qv.Rotary()
    k, v = _rows(sum(lens), hkv, seed=17)
    pos, cu = torch.zeros(sum(lens), dtype=torch.int32, device="cuda"), _cu(lens)

    def step(x):
        for layer in range(2):
            x.append(layer, k, v, cu, r, pos)
        x.advance(cu)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(bc)
        step(ref)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(bc)
    for i in range(6):
        k.copy_(_rows(sum(lens), hkv, seed=30 + i)[0])
        v.copy_(_rows(sum(lens), hkv, seed=40 + i)[1])
        pos.random_(0, 50000)
        g.replay()
        torch.cuda.synchronize()
        step(ref)
        for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "lens"):
            assert torch.equal(getattr(bc, name), getattr(ref, name)), (i, name)


def test_pages_and_rows_past_2_to_the_31():
    """Pages whose codes begin past 2^31 bytes, rows further than 2^31 elements apart."""
    import paper_2608_05326_amd as qv
    import torch
    hkv, T, st = 4, 700, 1 << 22
    pages = (1 << 31) // (hkv * N * D) + 40
    bc = qv.BlockCache(qv.BlockConfig(1, 4, hkv, 1000, num_pages=pages))
    bc.table = torch.arange(pages - 16, pages, dtype=torch.int32)[None]
    bc.lens = torch.tensor([33], dtype=torch.int32)
    bc.k_tail.copy_(_bf16(1, 1, hkv, N, D, seed=18))
    bc.v_tail.copy_(_bf16(1, 1, hkv, N, D, seed=19))
    buf = torch.empty((T - 1) * st + hkv * D, dtype=torch.bfloat16, device="cuda")
    k = buf.as_strided((T, hkv, D), (st, D, 1))
    k.copy_(_bf16(T, hkv, D, seed=20))
    v = _bf16(T, hkv, D, seed=21).cuda()
    tails = bc.k_tail[0, 0].clone(), bc.v_tail[0, 0].clone()
    bc.append(0, k, v, _cu([T]))
    rows = [torch.cat([t[:, :33], x.transpose(0, 1)], 1) for t, x in zip(tails, (k, v))]
    for b in range((33 + T) // N):
        _check_closed(bc, 0, 0, b, *[x[:, b * N:(b + 1) * N] for x in rows])
    assert torch.equal(bc.k_tail[0, 0, :, :(33 + T) % N], rows[0][:, (33 + T) // N * N:])


def test_on_a_stream_of_its_own():
    import paper_2608_05326_amd as qv
    import torch
    held, lens, hkv = [50, 10], [30, 200], 2
    want = _fresh(held, hkv, 300, seed=22)
    k, v = _rows(sum(lens), hkv, seed=23)
    want.append(0, k, v, _cu(lens))
    want.advance(_cu(lens))
    side = torch.cuda.Stream()
    cfg = qv.BlockConfig(2, 4, hkv, want.cfg.max_context, num_pages=want.num_pages)
    torch.cuda.synchronize()
    bc = qv.BlockCache(cfg, stream=side)
    start = _fresh(held, hkv, 300, seed=22)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "lens"):
        setattr(bc, name, getattr(start, name))
    cu = _cu(lens)
    side.wait_stream(torch.cuda.current_stream())
    bc.append(0, k, v, cu)
    bc.advance(cu)
    side.synchronize()
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "lens"):
        assert torch.equal(getattr(bc, name), getattr(want, name)), name
