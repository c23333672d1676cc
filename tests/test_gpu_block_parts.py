"""Decode steps of the block cache whose parts hold many blocks: several waves in a segment,
parts that cross KV heads and places, joins of them, layers past the caches, and more than 64
blocks a wave.  Against float64 on the CPU; tolerances as in test_gpu_block_cache.py but where
a test derives its own."""
import numpy as np
import pytest
from test_gpu_block_cache import _bf16, _make, _step

pytestmark = pytest.mark.gpu
D, N = 128, 64
PARTS, COST, SMALL = 480, 4, 8      # qv_parts.h


def _part(lens, hkv, max_context=1 << 40):
    """Items of a part: blocks and cost of the pairs that are split."""
    n = [t // N for t in lens if 0 <= t < max_context]
    return -(-sum(b + COST for b in n if b > SMALL) * hkv // PARTS)


LENS = [2500, 4095, -1, 3200, 63, 6001, 576, 575, 0, 1300]


@pytest.mark.parametrize("hq,hkv,part", [(4, 4, 3), (8, 8, 5), (32, 16, 10)])
@pytest.mark.parametrize("large", [False, True])
def test_parts_of_several_blocks(hq, hkv, part, large):
    """Ragged places, every eighth page dropped (whole runs of a segment among them); a large
    layer is read past the caches (the one of 16 heads is large without spare pages)."""
    import torch
    bc, _, _ = _make(LENS, hq, hkv, seed=hkv, spare=8400 // hkv if large else 2)
    assert _part(LENS, hkv) == part
    assert (bc.num_pages * hkv * 2 * N * D > 128 << 20) == (large or hkv == 16)
    bc.table[:, 3::8] = -1
    bc.table[3, 8:30] = -1
    bc.table[5, 40:52] = 1 << 20
    q, kn, vn, out = _step(bc, LENS, seed=70 + hkv)
    again = torch.full_like(out, 7.0)
    bc.attend(0, q, kn, vn, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("places", [64, 150])
def test_parts_across_places(places):
    """Places of 9 to 24 blocks and short ones between them: a part crosses several places,
    also past the 64 that a wave counts at once."""
    rng = np.random.default_rng(places)
    lens = rng.integers(560, 1550, places)
    lens[::7] = rng.integers(-1, 300, len(lens[::7]))
    lens = lens.tolist()
    assert _part(lens, 4) > 4 * (places // 32)
    bc, _, _ = _make(lens, 8, 4, seed=places)
    _step(bc, lens, seed=80)


def test_steps_with_parts_across_block_ends():
    """Steps on which the parts' sizes and a pair's number of blocks change."""
    lens = [1980, 575, 4090, 638, 3000]
    bc, _, _ = _make(lens, 16, 16, seed=81)
    for t in range(5):
        _step(bc, lens, seed=82 + 3 * t)
        bc.advance()
        lens = [x + 1 for x in lens]
        assert _part(lens, 16) > 4


@pytest.mark.parametrize("spare", [0, 460])
def test_more_than_64_blocks_a_wave(spare):
    """One place of 16384 blocks, 16 KV heads: 547 items a part, so that a wave asks three
    times for 64 pages.  The blocks share a few pages (read only); 48 of them have a page of
    their own, whose keys follow the query, so that each of those holds about 1% of every
    row's weight and is missed if it is left out or counted twice.

    Tolerance: a probability is off by 2^-11 of itself or 2^-25 of the largest (fp16), in the
    open block by 2^-8 (bf16); a logit by 130 x 2^-24 sum|q k| scale (128 products and two
    factors), which enters twice; fewer than 2^12 fp32 sums in numerator and denominator, 2^-12
    each; the exponentials 2^-22; the output 2^-8."""
    import torch
    import paper_2608_05326_amd as qv
    n_blk, hkv, G, common, own = 16384, 16, 2, 24, 48
    t = n_blk * N + 5
    assert _part([t], hkv) == 547
    g = torch.Generator().manual_seed(90)
    pages = common + own + spare
    bc = qv.BlockCache(qv.BlockConfig(1, G * hkv, hkv, t + 10, num_pages=pages))
    assert (pages * hkv * 2 * N * D > 128 << 20) == (spare > 0)
    base = torch.randn(hkv, D, generator=g)
    q = (base[:, None] + 0.2 * torch.randn(hkv, G, D, generator=g)).bfloat16()      # [hkv, G, D]
    kc = torch.randint(-127, 128, (pages, hkv, N, D), generator=g)
    vc = torch.randint(-127, 128, (pages, hkv, D, N), generator=g)
    ks, vs = torch.full((pages, hkv), 0.5 / 70), torch.full((pages, hkv), 1.0 / 70)
    mine = torch.arange(common, common + own)
    dirs = base / base.abs().amax(dim=1, keepdim=True) * 127
    noise = torch.randint(-20, 21, (own, hkv, N, D), generator=g)
    kc[mine] = (dirs[None, :, None] + noise).round().clamp(-127, 127).long()
    # logit about 6.2: exp of it times 48 x 64 tokens is the weight of the other million
    ks[mine] = (6.2 * D ** 0.5 / (dirs * base).sum(1))[None]
    vc[mine] = torch.randint(-127, 128, (own, hkv, D, 1), generator=g).expand(-1, -1, -1, N)
    vs[mine] = 4.0 / 70
    table = torch.randint(0, common, (n_blk + 1,), generator=g)
    table[torch.rand(n_blk + 1, generator=g) < 0.05] = -1
    at = torch.randperm(n_blk, generator=g)[:own]
    table[at] = mine
    bc.k_codes, bc.v_codes = kc[None].to(torch.int8), vc[None].to(torch.int8)
    bc.k_scale, bc.v_scale = ks[None], vs[None]
    bc.table, bc.lens = table[None].int(), torch.tensor([t], dtype=torch.int32)
    tail = _bf16(2, hkv, N, D, seed=91)
    bc.k_tail, bc.v_tail = tail[0][None, None], tail[1][None, None]
    kn, vn = _bf16(1, hkv, D, seed=92), _bf16(1, hkv, D, seed=93)
    out = torch.zeros(1, G * hkv, D, dtype=torch.bfloat16, device="cuda")
    qd = q.reshape(1, G * hkv, D).cuda()
    bc.attend(0, qd, kn.cuda(), vn.cuda(), out)
    again = torch.zeros_like(out)
    bc.attend(0, qd, kn.cuda(), vn.cuda(), again)
    got = out.double().cpu()
    assert torch.equal(out, again)

    count = torch.bincount(table[:n_blk][table[:n_blk] >= 0], minlength=pages).double()
    for h in range(hkv):
        kk = (kc[:, h].double() * ks[:, h].double().view(-1, 1, 1)).reshape(-1, D)
        vv = (vc[:, h].double() * vs[:, h].double().view(-1, 1, 1)).transpose(1, 2).reshape(-1, D)
        kk = torch.cat([kk, tail[0, h, :5].double(), kn[0, h].double()[None]])
        vv = torch.cat([vv, tail[1, h, :5].double(), vn[0, h].double()[None]])
        m = torch.cat([count.repeat_interleave(N), torch.ones(6, dtype=torch.float64)])
        half = torch.full_like(m, 2.0 ** -11)
        half[-6:] = 2.0 ** -8
        for j in range(G):
            x = q[h, j].double()
            s = (kk @ x) * D ** -0.5
            S = ((kk.abs() @ x.abs()) * D ** -0.5)[m > 0].max()
            e = torch.exp(s - s[m > 0].max())
            w = m * e
            L = w.sum()
            o, A = (w @ vv) / L, (w @ vv.abs()) / L
            E = ((m * torch.maximum(half * e, torch.tensor(2.0 ** -25, dtype=torch.float64))) @ vv.abs()) / L
            tol = 2.0 ** -8 * o.abs() + E + (260 * 2.0 ** -24 * S + 2.0 ** -11 + 2.0 ** -21) * A
            err = (got[0, h * G + j] - o).abs()
            assert bool((err <= tol).all()), (h, j, (err / tol).max().item())
            # a block of its own left out (or counted twice) would be seen
            for b in range(own):
                rows = slice((common + b) * N, (common + b + 1) * N)
                less = (w @ vv - w[rows] @ vv[rows]) / (L - w[rows].sum())
                assert bool(((less - o).abs() > 2 * tol).any()), (h, j, b)
