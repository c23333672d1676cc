"""The 8-bit block cache (store, attend, fetch) against float64 / exact arithmetic on the CPU.

Codes and scales are decided exactly, so they are compared for equality; a fetched value is
one fp32 product rounded to bf16, compared for equality too.

Tolerance of attention, per output element, with A = sum_j p_j |v_j| and n tokens: a
probability is rounded once, to fp16 (blocks: 2^-11 relative, at most 2^-25 of the largest
probability below fp16's normal range) or bf16 (open block: 2^-8), the output once to bf16
(2^-8); logits are fp32 sums of 128 exact products (2^-24 x 128 x sum |q k| scale, under
2^-12 for these inputs), which enters twice: |error| <= 2^-8 (A + |o|) + 2^-11 A
+ n 2^-25 max|v|."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
D, N = 128, 64


def _bf16(*shape, seed=0, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).bfloat16()


def _cu(lens):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()


def _quantize(x):
    """Block [64, d] bf16 -> (codes, scale), from the definition."""
    x = x.float().numpy()
    a = np.abs(x).max()
    if not np.isfinite(a):
        return np.zeros(x.shape, np.int8), np.float32(np.nan)
    s = max(np.float32(np.float64(a) / 127.0), np.float32(2.0 ** -100))
    # a bf16 over a fp32 lies off a half-integer by 2^-25 of it at least, or is one: a
    # float64 quotient rounds as the exact one
    return np.rint(x.astype(np.float64) / np.float64(s)).astype(np.int8), s


class Model:
    """What a cache holds, kept by the test: per place and head the values readers take."""

    def __init__(self, bc):
        self.bc, c = bc, bc.cfg
        self.vals = [[None] * c.num_kv_heads for _ in range(c.batch)]   # (k, v) float64 [n, d]

    def held(self, place, h, t):
        """Values of tokens 0 .. t - 1 read from the cache's own tensors."""
        import torch
        b = self.bc
        n = t // N
        pages = b.table[place, :n].cpu().tolist()
        ks, vs, keep = [], [], []
        for p in pages:
            ok = 0 <= p < b.num_pages
            keep += [ok] * N
            if ok:
                ks.append(b.k_codes[0, p, h].cpu().double() * b.k_scale[0, p, h].cpu().double())
                vs.append(b.v_codes[0, p, h].cpu().double().T * b.v_scale[0, p, h].cpu().double())
            else:
                ks.append(torch.zeros(N, D, dtype=torch.float64))
                vs.append(torch.zeros(N, D, dtype=torch.float64))
        r = t - n * N
        keep += [True] * r
        ks.append(b.k_tail[0, place, h, :r].cpu().double())
        vs.append(b.v_tail[0, place, h, :r].cpu().double())
        return torch.cat(ks), torch.cat(vs), torch.tensor(keep, dtype=torch.bool)


def _make(lens, hq, hkv, max_context=None, shuffle=True, seed=0, scale=1.0, layers=1, spare=2, fill=float("nan")):
    """A cache whose places hold prompts of the given lengths (-1: empty), pages in no
    order, unused tail rows and pages holding `fill`; returns (cache, k, v packed)."""
    import torch
    import paper_2608_05326_amd as qv
    mc = max_context or max(max(lens), 1) + 70
    cols = -(-mc // N)
    bc = qv.BlockCache(qv.BlockConfig(len(lens), hq, hkv, mc, num_layers=layers,
                                      num_pages=len(lens) * cols + spare if shuffle else 0))
    if shuffle:
        order = np.random.default_rng(seed).permutation(bc.num_pages)[:len(lens) * cols]
        bc.table = torch.from_numpy(order.astype(np.int32).reshape(len(lens), cols))
    bc.k_tail.fill_(fill)
    bc.v_tail.fill_(fill)
    bc.k_scale.fill_(fill)
    bc.v_scale.fill_(fill)
    pos = [max(t, 0) for t in lens]
    k, v = (_bf16(sum(pos), hkv, D, seed=seed + i, scale=scale).cuda() for i in (1, 2))
    for layer in range(layers):
        bc.store(layer, k, v, _cu(pos))
    bc.lens = torch.tensor(lens, dtype=torch.int32)
    return bc, k, v


def _attention(q, kk, vv, keep, scale=D ** -0.5):
    """q [d] float64: (o, A) over the kept tokens."""
    import torch
    s = (kk @ q) * scale
    p = torch.softmax(torch.where(keep, s, -torch.inf), 0)
    vz = torch.where(keep[:, None], vv, 0.0)
    return p @ vz, p @ vz.abs(), vz.abs().max()


def _step(bc, lens, seed, scale=1.0, layer=0, check=True):
    """One attend at the given lengths, checked against the cache's own contents."""
    import torch
    c = bc.cfg
    q = _bf16(c.batch, c.num_q_heads, D, seed=seed, scale=scale).cuda()
    kn, vn = (_bf16(c.batch, c.num_kv_heads, D, seed=seed + i).cuda() for i in (1, 2))
    m = Model(bc)
    before = {(s, h): m.held(s, h, t) for s, t in enumerate(lens) for h in range(c.num_kv_heads)
              if 0 <= t < c.max_context}
    tails = bc.k_tail[layer].clone(), bc.v_tail[layer].clone()
    out = torch.full_like(q, 7.0)
    bc.attend(layer, q, kn, vn, out)
    torch.cuda.synchronize()
    if not check:
        return q, kn, vn, out
    got = out.double().cpu()
    qd = q.double().cpu()
    G = c.num_q_heads // c.num_kv_heads
    for s, t in enumerate(lens):
        if not 0 <= t < c.max_context:
            assert bool((out[s] == 7.0).all())
            continue
        for h in range(c.num_kv_heads):
            kk, vv, keep = before[s, h]
            kk = torch.cat([kk, kn[s, h].double().cpu()[None]])
            vv = torch.cat([vv, vn[s, h].double().cpu()[None]])
            keep = torch.cat([keep, torch.ones(1, dtype=torch.bool)])
            for j in range(h * G, h * G + G):
                o, A, vmax = _attention(qd[s, j], kk, vv, keep)
                tol = 2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A + (t + 1) * 2.0 ** -25 * vmax
                err = (got[s, j] - o).abs()
                # (an open block that was never filled holds NaN: so does the result)
                ok = (err <= tol) | (got[s, j].isnan() & o.isnan())
                assert bool(ok.all()), (s, t, j, (err / tol).max().item())
        # the appended token, and nothing else, in the open block
        for tail, old, new in ((bc.k_tail, tails[0], kn), (bc.v_tail, tails[1], vn)):
            old[s, :, t % N] = new[s]
            assert torch.equal(tail[layer, s].view(torch.int16), old[s].view(torch.int16))
        if t % N == N - 1:
            _check_closed(bc, layer, s, t // N, bc.k_tail[layer, s], bc.v_tail[layer, s])
    return q, kn, vn, out


def _check_closed(bc, layer, place, blk, k, v):
    """Page of a complete block against k, v [H_kv, 64, d]."""
    p = int(bc.table[place, blk])
    if not 0 <= p < bc.num_pages:
        return
    for h in range(bc.cfg.num_kv_heads):
        for x, codes, sc in ((k, bc.k_codes[layer, p, h], bc.k_scale), (v, bc.v_codes[layer, p, h].T, bc.v_scale)):
            want, s = _quantize(x[h].cpu())
            got = sc[layer, p, h].cpu().numpy()
            assert got == s or (np.isnan(got) and np.isnan(s))
            assert np.array_equal(codes.cpu().numpy(), want)


@pytest.mark.parametrize("lens", [[1], [63], [64], [65], [128, 1, 0, 200], [5] * 70, [777]],
                         ids=lambda x: "-".join(map(str, x[:5])))
@pytest.mark.parametrize("hkv", [1, 3])
def test_store_and_fetch(lens, hkv):
    import torch
    bc, k, v = _make(lens, 2 * hkv, hkv, seed=len(lens))
    cu = np.concatenate([[0], np.cumsum(lens)])
    for s, t in enumerate(lens):
        a = int(cu[s])
        for b in range(t // N):
            rows = slice(a + b * N, a + (b + 1) * N)
            _check_closed(bc, 0, s, b, k[rows].transpose(0, 1), v[rows].transpose(0, 1))
        r = t % N
        for tail, x in ((bc.k_tail, k), (bc.v_tail, v)):
            assert torch.equal(tail[0, s, :, :r], x[a + t - r:a + t].transpose(0, 1))
            assert bool(tail[0, s, :, r:].isnan().all())          # untouched
    ko, vo = (torch.full_like(k, 7.0) for _ in range(2))
    bc.fetch(0, ko, vo, _cu(lens))
    m = Model(bc)
    for s, t in enumerate(lens):
        for h in range(hkv):
            kk, vv, _ = m.held(s, h, t)
            for got, want in ((ko, kk), (vo, vv)):
                # code x scale in float64 is exact; fp32 then bf16
                assert torch.equal(got[cu[s]:cu[s + 1], h].cpu(), want.float().bfloat16())


def test_codes_at_ties_and_extremes():
    """Exact half steps, the type's largest and smallest values, zeros, one outlier."""
    import torch
    import paper_2608_05326_amd as qv
    blocks = []
    x = torch.zeros(N, D)
    x[0, 0] = 127.0
    x[1] = torch.arange(D) - 64 + 0.5                   # ties at scale 1
    x[2] = -x[1]
    blocks.append(x)
    x = torch.randn(N, D, generator=torch.Generator().manual_seed(0))
    blocks += [x * 2.0 ** 100, x * 2.0 ** -96, x * 2.0 ** -120, x * 1e-38, torch.zeros(N, D),
               torch.full((N, D), 3.3895e38), torch.full((N, D), 9.2e-41)]
    y = x.clone()
    y[17, 3] = 1e30
    blocks.append(y)
    y = x.clone()
    y[17, 3] = -65504.0
    blocks.append(y)
    for bad in (float("inf"), float("-inf"), float("nan")):
        y = x.clone()
        y[63, 127] = bad
        blocks.append(y)
    k = torch.cat(blocks).bfloat16()[:, None].cuda()
    v = k.flip(0).contiguous()
    n = len(blocks)
    bc = qv.BlockCache(qv.BlockConfig(1, 1, 1, n * N))
    bc.store(0, k, v, _cu([n * N]))
    torch.cuda.synchronize()
    for b in range(n):
        rows = slice(b * N, (b + 1) * N)
        _check_closed(bc, 0, 0, b, k[rows].transpose(0, 1), v[rows].transpose(0, 1))
    # half a step at most, by the codes that are there
    for b in range(n - 3):
        e = (k[b * N:(b + 1) * N, 0].double().cpu() -
             bc.k_codes[0, b, 0].cpu().double() * bc.k_scale[0, b, 0].cpu().double()).abs().max()
        # (the largest value is 127 s up to the rounding of s: 127 x 2^-24 relative)
        s = bc.k_scale[0, b, 0].cpu().double()
        assert e <= s / 2 * (1 + 2.0 ** -16)
    bc.lens.fill_(n * N)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    bc.fetch(0, ko, vo, _cu([n * N]))
    assert bool(ko[(n - 3) * N:].isnan().all()) and bool(ko[:(n - 3) * N].isfinite().all())


@pytest.mark.parametrize("lens", [[0], [1], [62], [63], [64], [127], [128, -1, 300, 0, 63], [1000], [3] * 40],
                         ids=lambda x: "-".join(map(str, x[:5])))
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (5, 1), (14, 2), (16, 1)])
def test_attend(lens, hq, hkv):
    bc, _, _ = _make(lens, hq, hkv, seed=hq)
    _step(bc, lens, seed=hq + len(lens))


@pytest.mark.parametrize("lens", [[5000], [4095, 17, 2500], [9000, 63]])
def test_attend_longer(lens):
    bc, _, _ = _make(lens, 8, 2, seed=3)
    _step(bc, lens, seed=4, scale=2.0)


def test_many_places():
    """300 places (more than a wave's 64 lanes count at once), some empty, a few long."""
    rng = np.random.default_rng(7)
    lens = rng.integers(-1, 40, 300)
    lens[[5, 63, 64, 130, 299]] = [900, 640, 639, 1100, 575]
    lens = lens.tolist()
    bc, k, v = _make(lens, 2, 1, seed=34)
    _step(bc, lens, seed=35)
    import torch
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    pos = [max(t, 0) for t in lens]
    bc.fetch(0, ko, vo, _cu(pos))
    a = sum(pos[:130])
    assert torch.equal(ko[a + 1088:a + 1100], k[a + 1088:a + 1100])   # place 130's open block
    assert bool(((ko.float() - k.float()).abs() <= 0.05).all())       # scales: 5 / 127, half a step and a rounding


def test_steps_across_block_ends():
    """70 steps of places at different lengths, blocks closing on the way."""
    import torch
    lens = [0, 60, 127, -1, 33]
    bc, _, _ = _make(lens, 4, 2, max_context=260, seed=21)
    for t in range(70):
        _step(bc, lens, seed=100 + 3 * t)
        bc.advance()
        lens = [x + 1 if x >= 0 else x for x in lens]
        assert bc.lens.cpu().tolist() == lens
    ko, vo = (torch.full((sum(max(x, 0) for x in lens), 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
              for _ in range(2))
    bc.fetch(0, ko, vo, _cu([max(x, 0) for x in lens]))
    assert bool(ko.isfinite().all()) and bool(vo.isfinite().all())


def test_places_without_room_or_sequence():
    import torch
    lens = [100, -1, 130, 129]
    bc, _, _ = _make([100, -1, 130, 129], 4, 2, max_context=130, seed=5)
    _step(bc, lens, seed=6)      # place 2 is full: skipped
    bc.advance()
    assert bc.lens.cpu().tolist() == [101, -1, 130, 130]
    bc.lens = torch.tensor([-7, 1 << 30, -(1 << 31), 131], dtype=torch.int32)
    q, kn, vn, out = _step(bc, [-1] * 4, seed=7, check=False)
    assert bool((out == 7.0).all())


def test_fetch_of_places_without_a_sequence():
    """Lengths below zero hold nothing, whatever rows cu_tokens gives them."""
    import torch
    bc, k, v = _make([200, 70, 130], 4, 2, max_context=300, seed=36)
    bc.lens = torch.tensor([-1, -(1 << 31), 1 << 30], dtype=torch.int32)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    bc.fetch(0, ko, vo, _cu([200, 70, 130]))
    assert bool((ko[:270] == 7.0).all()) and bool((vo[:270] == 7.0).all())
    assert bool((ko[270:398] != 7.0).any(-1).all())      # a length past max_context counts as max_context


@pytest.mark.parametrize("drop", [-1, 1 << 30, -(1 << 31)])
def test_blocks_without_a_page(drop):
    """Dropped blocks take no part, are not stored and are fetched as zeros."""
    import torch
    lens = [640, 64, 300]
    bc, k, v = _make(lens, 8, 2, seed=8)
    for s, b in ((0, 0), (0, 4), (0, 9), (1, 0), (2, 1), (2, 2), (2, 3)):
        bc.table[s, b] = drop
    _step(bc, lens, seed=9)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    bc.fetch(0, ko, vo, _cu(lens))
    assert bool((ko[:N] == 0).all()) and bool((vo[4 * N:5 * N] == 0).all())
    assert bool((ko[640:704] == 0).all()) and bool((ko[N:2 * N] != 0).any())
    codes, scales = bc.k_codes.clone(), bc.k_scale.clone()
    bc.store(0, k.flip(0), v.flip(0), _cu(lens))
    gone = bc.num_pages - len(torch.unique(bc.table[(bc.table >= 0) & (bc.table < bc.num_pages)]))
    same = (bc.k_codes == codes).flatten(2).all(2)[0]
    assert int(same.sum()) >= gone
    # a token that fills a block without a page: nothing is written
    bc.table[1, 0] = drop
    bc.lens[1] = 63
    codes = bc.k_codes.clone(), bc.v_codes.clone()
    bc.lens[0] = bc.lens[2] = -1
    _step(bc, [-1, 63, -1], seed=10)
    assert torch.equal(bc.k_codes, codes[0]) and torch.equal(bc.v_codes, codes[1])


def test_every_block_without_a_page():
    lens = [192, 5]
    bc, _, _ = _make(lens, 4, 1, seed=11)
    bc.table.fill_(-1)
    _step(bc, lens, seed=12)


def test_values_that_are_not_finite():
    """Stale rows past the new token never count; a NaN block makes its head's rows NaN only."""
    import torch
    lens = [130, 130]
    bc, _, _ = _make(lens, 4, 2, seed=13)       # pages and rows that are not in use hold NaN
    p = int(bc.table[0, 1])
    bc.v_scale[0, p, 1] = float("nan")
    q, kn, vn, out = _step(bc, lens, seed=14, check=False)
    assert bool(out[0, 2:].isnan().all()) and bool(out[0, :2].isfinite().all()) and bool(out[1].isfinite().all())
    bc.v_scale[0, p, 1] = 1.0
    bc.k_scale[0, p, 0] = float("nan")
    q, kn, vn, out = _step(bc, lens, seed=14, check=False)
    assert bool(out[0, :2].isnan().all()) and bool(out[0, 2:].isfinite().all()) and bool(out[1].isfinite().all())
    bc.k_scale[0, p, 0] = 1.0
    kn[0, 0, 5] = float("inf")
    q[0, 3, 7] = float("nan")
    bc.attend(0, q, kn, vn, out)
    assert bool(out[0, :2].isnan().any()) and bool(out[0, 3].isnan().all()) and bool(out[0, 2].isfinite().all())
    assert bool(out[1].isfinite().all())


def test_scales_far_apart_and_large_queries():
    """Blocks whose values differ by 2^40, and queries at the ends of bf16's range."""
    import torch
    lens = [320]
    bc, _, _ = _make(lens, 4, 1, seed=15)
    pages = bc.table[0, :5].long()
    bc.v_scale[0, pages, 0] = torch.tensor([1e-8, 1e4, 1.0, 1e-4, 3e3], device="cuda")
    _step(bc, lens, seed=16)
    for f in (2.0 ** 60, 2.0 ** -60):
        bc2, _, _ = _make(lens, 4, 1, seed=17)
        bc2.k_scale.mul_(1.0 / f)
        bc2.k_tail.mul_(1.0 / f)
        q = (_bf16(1, 4, D, seed=18).double() * f).bfloat16().cuda()
        kn = (_bf16(1, 1, D, seed=19).double() / f).bfloat16().cuda()
        vn = _bf16(1, 1, D, seed=20).cuda()
        m = Model(bc2)
        kk, vv, keep = m.held(0, 0, 320)
        out = torch.zeros_like(q)
        bc2.attend(0, q, kn, vn, out)
        kk = torch.cat([kk, kn[0, 0].double().cpu()[None]])
        vv = torch.cat([vv, vn[0, 0].double().cpu()[None]])
        for j in range(4):
            o, A, vmax = _attention(q[0, j].double().cpu(), kk, vv, torch.ones(321, dtype=torch.bool))
            err = (out[0, j].double().cpu() - o).abs()
            assert bool((err <= 2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A + 321 * 2.0 ** -25 * vmax).all())


def test_strides_of_packed_rows():
    import torch
    lens = [100, 64, 29]
    x = _bf16(sum(lens), 12, D, seed=22).cuda()          # fused rows: 8 query, 2 key, 2 value heads
    a, k, v = _make(lens, 8, 2, seed=23)
    a.store(0, x[:, 8:10], x[:, 10:], _cu(lens))
    b, _, _ = _make(lens, 8, 2, seed=23)
    kt, vt = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (x[:, 8:10], x[:, 10:]))
    b.store(0, kt, vt, _cu(lens))
    for n in ("k_codes", "v_codes"):
        assert torch.equal(getattr(a, n), getattr(b, n))
    big = torch.full((sum(lens), 6, D), 7.0, dtype=torch.bfloat16, device="cuda")
    a.fetch(0, big[:, 1:3], big[:, 4:6], _cu(lens))
    k0, v0 = torch.zeros_like(k), torch.zeros_like(v)
    b.fetch(0, k0, v0, _cu(lens))
    assert torch.equal(big[:, 1:3], k0) and torch.equal(big[:, 4:6], v0)
    assert bool((big[:, [0, 3]] == 7.0).all())


def test_store_leaves_other_places_and_limits():
    """A store of one place, rows past max_context, fetches of fewer and more tokens than held."""
    import torch
    lens = [100, 70, 200]
    bc, k, v = _make(lens, 4, 2, max_context=200, seed=24)
    keep = {n: getattr(bc, n).clone() for n in ("k_codes", "v_codes", "k_tail", "v_tail", "k_scale")}
    k2, v2 = (_bf16(300, 2, D, seed=25 + i).cuda() for i in (0, 1))
    bc.store(0, k2, v2, _cu([0, 300, 0]))                 # 100 rows too many
    mine = bc.table[1, :4].long()
    for n in ("k_codes", "v_codes", "k_scale"):
        x, y = getattr(bc, n)[0], keep[n][0]
        other = torch.ones(bc.num_pages, dtype=torch.bool, device="cuda")
        other[mine] = False
        assert torch.equal(x[other].nan_to_num(0), y[other].nan_to_num(0))
    for n in ("k_tail", "v_tail"):
        for s in (0, 2):
            assert torch.equal(getattr(bc, n)[0, s].view(torch.int16), keep[n][0, s].view(torch.int16))
    assert torch.equal(bc.k_tail[0, 1, :, :8], k2[192:200].transpose(0, 1))
    bc.lens = torch.tensor([100, 200, -1], dtype=torch.int32)
    ko, vo = (torch.full((30 + 250 + 5, 2, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bc.fetch(0, ko, vo, _cu([30, 250, 5]))
    assert bool((ko[230:] == 7.0).all()) and bool((vo[230:] == 7.0).all())
    assert torch.equal(ko[30 + 192:230], k2[192:200])
    assert bool((ko[:230] != 7.0).any(-1).all())


def test_layers_are_independent():
    import torch
    lens = [130, 63]
    bc, k, v = _make(lens, 4, 2, layers=3, seed=26)
    was = bc.k_tail[[0, 2]].clone(), bc.k_codes[[0, 2]].clone()
    q, kn, vn, out = _step(bc, lens, seed=27, layer=1, check=False)
    assert torch.equal(bc.k_tail[[0, 2]].view(torch.int16), was[0].view(torch.int16))
    assert torch.equal(bc.k_codes[[0, 2]], was[1])
    out2 = torch.zeros_like(out)
    bc.attend(2, q, kn, vn, out2)
    assert torch.equal(out, out2)
    for bad in (-1, 3):
        with pytest.raises(ValueError):
            bc.attend(bad, q, kn, vn, out)


def test_repeats_bitwise_and_on_another_stream():
    import torch
    lens = [3000, 20, 1500, 63]
    bc, _, _ = _make(lens, 8, 2, seed=28)
    q, kn, vn, out = _step(bc, lens, seed=29)
    page = int(bc.table[3, 0])
    codes = bc.k_codes[0, page].clone()
    st = torch.cuda.Stream()
    for _ in range(3):
        again = torch.zeros_like(out)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            bc.attend(0, q, kn, vn, again)
        st.synchronize()
        assert torch.equal(out, again) and torch.equal(bc.k_codes[0, page], codes)


def test_captured_steps():
    """A step and its advance captured once, replayed across block ends, against the eager
    steps of a second cache."""
    import torch
    lens = [60, 0, 127, -1, 500]
    a, _, _ = _make(lens, 8, 2, max_context=640, seed=30)
    b, _, _ = _make(lens, 8, 2, max_context=640, seed=30)
    q, kn, vn = (_bf16(5, h, D, seed=31 + h).cuda() for h in (8, 2, 2))
    oa, ob = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    a.attend(0, q, kn, vn, oa)      # the same step again below
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.attend(0, q, kn, vn, oa)
        a.advance()
    for t in range(10):
        for x, s in ((q, 40), (kn, 41), (vn, 42)):
            x.copy_(_bf16(*x.shape, seed=s + 3 * t))
        graph.replay()
        b.attend(0, q, kn, vn, ob)
        b.advance()
        torch.cuda.synchronize()
        assert torch.equal(oa, ob) and torch.equal(a.lens, b.lens), t
    for n in ("k_codes", "v_codes", "k_tail", "v_tail"):
        x, y = getattr(a, n), getattr(b, n)
        assert torch.equal(x.view(torch.int8), y.view(torch.int8))


def test_refusals():
    import torch
    import paper_2608_05326_amd as qv
    bc, k, v = _make([100, 30], 8, 2, seed=33)
    q, kn, vn = (torch.zeros(2, h, D, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    for bad in (dict(q=q.float()), dict(kn=kn.cpu()), dict(vn=vn[:1]), dict(out=q[:, ::2]), dict(q=q[:, :4])):
        a = dict(q=q, kn=kn, vn=vn, out=torch.zeros_like(q))
        a.update(bad)
        with pytest.raises(ValueError):
            bc.attend(0, a["q"], a["kn"], a["vn"], a["out"])
    cu = _cu([100, 30])
    for a in ((k.float(), v, cu), (k, v[:-1], cu), (k[:, :1], v, cu), (k, v, cu[:2].contiguous()), (k, v, cu.long()),
              (k.cpu(), v, cu), (k[..., :64], v[..., :64], cu)):
        for call in (bc.store, bc.fetch):
            with pytest.raises(ValueError):
                call(0, *a)
    with pytest.raises(qv.QEvictError):
        bc.fetch(0, k[:, :1].expand(-1, 2, -1), v, cu)
    for cfg in (qv.BlockConfig(0, 8, 2, 100), qv.BlockConfig(1, 8, 2, 0)):
        with pytest.raises(ValueError):
            qv.BlockCache(cfg)


def test_prompts_through_both_caches():
    """A serving program's path: prompt attention, the block cache, decode steps, and the
    tiered cache taking a sequence over from it."""
    import torch
    import paper_2608_05326_amd as qv
    lens, hq, hkv = [200, 96, 333], 8, 2
    x = _bf16(sum(lens), hq + 2 * hkv, D, seed=50).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    cu = _cu(lens)
    prompt_out = qv.prompt_attend(q, k, v, cu)
    bc = qv.BlockCache(qv.BlockConfig(3, hq, hkv, 512))
    bc.store(0, k, v, cu)
    bc.lens = torch.tensor(lens, dtype=torch.int32)
    # a decode step with a prompt's last token in place of a new one repeats its row, up to
    # the cache's half steps: o changes by at most 2 A dl + the values' half step
    last = torch.tensor([199, 295, 628], device="cuda")
    bc.lens -= 1
    kt, vt = bc.k_tail[0].clone(), bc.v_tail[0].clone()
    out = torch.zeros(3, hq, D, dtype=torch.bfloat16, device="cuda")
    for s in range(3):   # the open block as it was before the last token
        if lens[s] % N == 0:
            pytest.fail("pick lengths inside a block")
    bc.attend(0, q[last].contiguous(), k[last].contiguous(), v[last].contiguous(), out)
    assert torch.equal(bc.k_tail[0], kt) and torch.equal(bc.v_tail[0], vt)
    step = max(bc.k_scale.max().item(), bc.v_scale.max().item())
    for s in range(3):
        for j in range(hq):
            qq = q[last[s], j].double().cpu()
            dl = step / 2 * qq.abs().sum().item() * D ** -0.5     # a logit's error
            vmax = v.abs().max().item()
            tol = 2 * np.expm1(dl) * vmax + step / 2 + 2.0 ** -7 * vmax
            assert (out[s, j] - prompt_out[last[s], j]).abs().max().item() <= tol
    bc.advance()
    # sequence 2 moves to the tiered cache
    ko, vo = (torch.zeros(333, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bc.fetch(0, ko, vo, _cu([0, 0, 333]))
    cfg = qv.Config(batch=1, num_q_heads=hq, num_kv_heads=hkv, window_tokens=32, quant_bits=4, max_context=512,
                    capacity_full=16, capacity_quant=0, out_dtype=qv.OUT_BF16)
    tier = qv.Cache(cfg)
    kk, vv = (t.transpose(0, 1).contiguous()[None] for t in (ko, vo))
    obs = q[-32:].transpose(0, 1).contiguous()[None]
    tier.prefill_assign(0, kk, vv, tier.prefill_scores(obs, kk))
    qn, kn, vn = (_bf16(3, h, D, seed=60 + h).cuda() for h in (hq, hkv, hkv))
    full = torch.zeros(1, hq, D, dtype=torch.bfloat16, device="cuda")
    tier.decode_attend(0, qn[2:3].contiguous(), kn[2:3].contiguous(), vn[2:3].contiguous(), full)
    bc.attend(0, qn, kn, vn, out)
    # the same keys and values up to the bf16 rounding of the fetched ones (every window
    # Full in the tiered cache): 2^-8 relative in keys (logits) and values
    for j in range(hq):
        dl = 2.0 ** -8 * (kk.abs().max() * qn[2, j].abs().sum()).item() * D ** -0.5
        vmax = vv.abs().max().item()
        assert (out[2, j] - full[0, j]).abs().max().item() <= 2 * np.expm1(dl) * vmax + 3 * 2.0 ** -8 * vmax
    tier.close()
