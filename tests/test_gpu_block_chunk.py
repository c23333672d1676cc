"""Attention of chunks of new tokens over the block cache, against float64.

Tolerance, per output element, with A = sum_j p_j |v_j|: a weight is rounded once to bf16, by
2^-8 of itself, the output once to bf16 (2^-8); a logit is an fp32 sum of 128 products (2^-24 x
128 x sum |q k| scale, under 2^-12 for the inputs here) and enters twice, with the logarithm of
a block's scale and the running maximum (2^-24 of a few hundred):
|error| <= 2^-8 (A + |o|) + 2^-11 A.  A weight is an fp32 number relative to the row's largest:
one below 2^-126 of it (fp32's smallest normal number) may count as zero, which n keys bring to
n 2^-126 max |v| at most (where the heaviest key's value is zero, A may be as small)."""
import numpy as np
import pytest

from test_gpu_block_cache import D, N, _bf16, _cu, _make

pytestmark = pytest.mark.gpu


def _cache(held, hq, hkv, chunk, seed=0, extra=70, fill=float("nan"), **kw):
    """A cache whose places hold `held` tokens (-1: none), pages in no order, unused rows and
    pages holding `fill`."""
    import paper_2608_05326_amd as qv
    import torch
    base, _, _ = _make(held, hq, hkv, max_context=max(max(held), 1) + extra, seed=seed, fill=fill, **kw)
    bc = qv.BlockCache(qv.BlockConfig(len(held), hq, hkv, base.cfg.max_context, num_pages=base.num_pages,
                                      chunk_tokens=chunk))
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "lens"):
        setattr(bc, name, getattr(base, name))
    torch.cuda.synchronize()
    return bc


def _held(bc, s, h, t, layer=0):
    """float64 keys, values and whether they take part, of tokens 0 .. t - 1, on the GPU."""
    import torch
    n = t // N
    p = bc.table[s, :n].long()
    there = (p >= 0) & (p < bc.num_pages)
    p = torch.where(there, p, 0)
    k = bc.k_codes[layer, p, h].double() * bc.k_scale[layer, p, h].double()[:, None, None]
    v = bc.v_codes[layer, p, h].double().transpose(1, 2) * bc.v_scale[layer, p, h].double()[:, None, None]
    r = t - n * N
    return (torch.cat([k.reshape(-1, D), bc.k_tail[layer, s, h, :r].double()]),
            torch.cat([v.reshape(-1, D), bc.v_tail[layer, s, h, :r].double()]),
            torch.cat([there.repeat_interleave(N), torch.ones(r, dtype=torch.bool, device="cuda")]))


def _check(bc, held, lens, q, k, v, out, fill=7.0, scale=None, starts=None, layer=0, loose=1.0):
    """Every row of out: attention in float64 from the cache's own tensors."""
    import torch
    c = bc.cfg
    G = c.num_q_heads // c.num_kv_heads
    scale = scale or D ** -0.5
    starts = np.concatenate([[0], np.cumsum(lens)]) if starts is None else starts
    seen = torch.zeros(q.shape[0], dtype=torch.bool)
    for s, a in enumerate(held):
        n = 0 if a < 0 or a >= c.max_context else min(lens[s], c.max_context - a)
        if not n:
            continue
        r0 = int(starts[s])
        seen[r0:r0 + n] = True
        for h in range(c.num_kv_heads):
            kk, vv, keep = _held(bc, s, h, a, layer)
            kk = torch.cat([kk, k[r0:r0 + n, h].double()])
            vv = torch.cat([vv, v[r0:r0 + n, h].double()])
            keep = torch.cat([keep, torch.ones(n, dtype=torch.bool, device="cuda")])
            vv = torch.where(keep[:, None], vv, 0.0)
            mask = keep[None] & (torch.arange(a + n, device="cuda")[None] <= torch.arange(a, a + n, device="cuda")[:, None])
            for j in range(h * G, h * G + G):
                w = q[r0:r0 + n, j].double() @ kk.t().contiguous() * scale
                p = torch.softmax(torch.where(mask, w, -torch.inf), 1)
                fin = torch.where(vv.isfinite(), vv, 0.0)
                o, A = p @ fin, p @ fin.abs()
                if not bool(vv.isfinite().all()):      # a row takes what is not finite where it sees it
                    for key in (~vv.isfinite().all(1)).nonzero().flatten().tolist():
                        bad = torch.where(vv[key].isfinite(), 0.0, vv[key])
                        o = o + torch.where(mask[:, key:key + 1], bad[None], 0.0)
                got = out[r0:r0 + n, j].double()
                tol = loose * (2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A) + (a + n) * 2.0 ** -126 * fin.abs().max()
                err = (got - o).abs()
                ok = (err <= tol) | (got.isnan() & o.isnan()) | (got == o)
                assert bool(ok.all()), (s, a, n, j, (~ok).nonzero()[:3].tolist(), (err / tol).nan_to_num(0).max().item())
    if fill is not None:
        assert bool((out.cpu()[~seen] == fill).all())


def _rows(T, hq, hkv, seed, scale=1.0):
    return (_bf16(T, hq, D, seed=seed, scale=scale).cuda(), _bf16(T, hkv, D, seed=seed + 1).cuda(),
            _bf16(T, hkv, D, seed=seed + 2).cuda())


def _run(bc, held, lens, seed=1, scale=1.0, **kw):
    import torch
    c = bc.cfg
    q, k, v = _rows(sum(lens), c.num_q_heads, c.num_kv_heads, seed, scale)
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    torch.cuda.synchronize()
    _check(bc, held, lens, q, k, v, out, **kw)
    return q, k, v, out


CASES = [
    ([0], [1]), ([0], [2]), ([0], [64]), ([0], [65]), ([0], [200]), ([1], [1]), ([63], [1]), ([63], [2]),
    ([64], [1]), ([64], [5]), ([65], [3]), ([127], [70]), ([640], [1]), ([1000], [4]), ([1000], [33]),
    ([200, -1, 0, 777, 64, 63, 5], [4, 3, 5, 1, 0, 17, 9]), ([130, 10], [300, 1]),
]


@pytest.mark.parametrize("held,lens", CASES, ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (5, 1), (14, 2), (16, 1), (3, 3)])
def test_chunk(held, lens, hq, hkv):
    _run(_cache(held, hq, hkv, sum(lens), seed=hq, extra=400), held, lens, seed=sum(lens))


@pytest.mark.parametrize("held,lens", [([5000], [7]), ([9000, 63, 4096], [3, 300, 1]), ([2500], [700]),
                                       ([4033, 4032, 4031], [64, 64, 64])])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (6, 1), (2, 2)])
def test_longer(held, lens, hq, hkv):
    _run(_cache(held, hq, hkv, sum(lens), seed=3, extra=800), held, lens, seed=4, scale=2.0)


# rows of a KV head at the ends of what a workgroup takes, and one past them
@pytest.mark.parametrize("rows", [31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1025])
@pytest.mark.parametrize("hq", [1, 3, 4, 7, 16])
def test_rows_of_a_workgroup(rows, hq):
    lens = [-(-rows // hq), max(rows // hq, 1)]
    _run(_cache([300, 1100], hq, 1, sum(lens), seed=rows, extra=1200), [300, 1100], lens, seed=rows + hq)


@pytest.mark.parametrize("held,lens", [([30001], [3]), ([30001], [9]), ([20000, 7], [60, 2]), ([12000, 9000], [1, 33]),
                                       ([1500], [100])])
@pytest.mark.parametrize("hq,hkv", [(6, 1), (2, 2)])
def test_many_parts(held, lens, hq, hkv):
    """Row tiles that many workgroups serve, with anything at all in the workspace."""
    bc = _cache(held, hq, hkv, sum(lens), seed=60)
    for byte in (0x7f, 0x80, 0xff, 0x01):
        bc.chunk_workspace.fill_(byte)
        _run(bc, held, lens, seed=61)


def test_many_places():
    """300 places (more than a wave's 64 lanes see at once), some empty, a few long."""
    rng = np.random.default_rng(7)
    held, lens = rng.integers(-1, 40, 300), rng.integers(0, 4, 300)
    held[[5, 63, 64, 130, 299]] = [900, 640, 639, 1100, 575]
    lens[[5, 63, 64, 131, 299]] = [3, 1, 70, 130, 2]
    held, lens = held.tolist(), lens.tolist()
    _run(_cache(held, 2, 1, sum(lens), seed=34, extra=200), held, lens, seed=35)


def test_a_token_is_a_decode_step():
    """One row for every place gives what attend gives (whose weights are rounded to fp16)."""
    import torch
    held = [0, 62, 63, 64, 1000, 129]
    bc = _cache(held, 8, 2, 6, seed=5)
    q, k, v, out = _run(bc, held, [1] * 6, seed=6)
    step = torch.zeros_like(q)
    bc.attend(0, q, k, v, step)
    size = out.double().abs().mean()
    assert (out.double() - step.double()).norm() <= 2.0 ** -7 * step.double().norm() and size > 0


def test_a_prompt_without_a_past_is_prompt_attend():
    import paper_2608_05326_amd as qv
    lens = [200, 1, 700, 0, 64]
    bc = _cache([0] * 5, 8, 2, sum(lens), seed=7, extra=800)
    q, k, v, out = _run(bc, [0] * 5, lens, seed=8)
    want = qv.prompt_attend(q, k, v, _cu(lens))
    assert (out.double() - want.double()).norm() <= 2.0 ** -7 * want.double().norm()


def test_strided_rows_and_rows_outside_the_places():
    """Slices of a projection, [H, T, d] tensors, an output with rows between; rows outside the
    places are neither read (NaN) nor written, bounds outside the rows are clamped."""
    import torch
    held, lens, hq, hkv = [100, 64, 30], [40, 3, 130], 8, 2
    T, starts = 300, [20, 60, 63]
    bc = _cache(held, hq, hkv, T, seed=9, extra=400)
    q, k, v = _rows(sum(lens), hq, hkv, seed=10)
    buf = torch.full((T, hq + 2 * hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[20:193, :hq], buf[20:193, hq:hq + hkv], buf[20:193, hq + hkv:] = q, k, v
    qs, ks, vs = buf[:, :hq], buf[:, hq:hq + hkv], buf[:, hq + hkv:]
    wide = torch.full((T, 2 * hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([20, 60, 63, 193], dtype=torch.int32).cuda()
    bc.attend_chunk(0, qs, ks, vs, cu, wide[:, 1::2])
    _check(bc, held, lens, qs, ks, vs, wide[:, 1::2], starts=starts)
    assert bool((wide[:, ::2] == 7.0).all())
    out = torch.full_like(q, 7.0)
    t = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    bc.attend_chunk(0, *t, torch.tensor([-9, 40, 43, 1 << 30], dtype=torch.int32).cuda(), out)
    assert torch.equal(out, wide[20:193, 1::2])


def test_room_and_places_without_a_sequence():
    import torch
    held = [100, -1, 130, 129, 66, 0]
    bc = _cache(held, 4, 2, 200, seed=11, extra=0)          # max_context 130
    assert bc.cfg.max_context == 130
    _run(bc, held, [40, 7, 3, 2, 64, 1], seed=12)
    bc.lens = torch.tensor([-7, 1 << 30, -(1 << 31), 131, 2 ** 31 - 1, 3], dtype=torch.int32)
    bc.k_tail.fill_(1.0)
    bc.v_tail.fill_(1.0)
    _run(bc, [-7, 1 << 30, -1, 131, 2 ** 31 - 1, 3], [40, 7, 3, 2, 64, 5], seed=13)
    # no place takes part: nothing is written
    bc.lens.fill_(-1)
    _run(bc, [-1] * 6, [40, 7, 3, 2, 64, 1], seed=14)


@pytest.mark.parametrize("drop", [-1, 1 << 30, -(1 << 31)])
def test_blocks_without_a_page(drop):
    held, lens = [640, 64, 300, 5000], [4, 70, 130, 9]
    bc = _cache(held, 8, 2, sum(lens), seed=15, extra=400)
    for s, b in ((0, 0), (0, 4), (0, 9), (1, 0), (2, 1), (2, 2), (2, 3)):
        bc.table[s, b] = drop
    bc.table[3, 5:70] = drop
    _run(bc, held, lens, seed=16)
    bc.table.fill_(drop)
    _run(bc, held, lens, seed=17)


def test_a_cache_without_pages():
    import paper_2608_05326_amd as qv
    import torch
    bc = qv.BlockCache(qv.BlockConfig(2, 4, 2, 500, num_pages=1, chunk_tokens=100))
    bc.lens = torch.tensor([0, 40], dtype=torch.int32)
    bc.k_tail.copy_(_bf16(1, 2, 2, N, D, seed=1))
    bc.v_tail.copy_(_bf16(1, 2, 2, N, D, seed=2))
    _run(bc, [0, 40], [70, 30], seed=18)


@pytest.mark.parametrize("lens", [[5, 6, 4], [150, 40, 70], [700, 3, 300]])
def test_values_that_are_not_finite(lens):
    """They reach the rows that see them: in the chunk, in an open block, in a page (whose scale
    is NaN then), in stale rows nowhere."""
    import torch
    held = [200, 300, 130]
    bc = _cache(held, 8, 2, sum(lens), seed=19, extra=800)
    q, k, v = _rows(sum(lens), 8, 2, seed=20)
    a1, a2 = lens[0], lens[0] + lens[1]
    v[3, 0, 5] = float("inf")
    v[2, 1, 77] = float("nan")
    v[a1 + 1, 1, 0] = float("-inf")
    v[a2 - 1, 0, 127] = float("inf")              # the last row of a place sees it alone
    bc.v_tail[0, 2, 0, 1, 9] = float("inf")
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    _check(bc, held, lens, q, k, v, out)
    # a key that is not finite, and masked ones
    k[a1 + 2, 0, 3] = float("nan")
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    rows = out[a1:a2, :4]
    assert bool(rows[2:].isnan().all()) and bool(out[a1:a2, 4:, 1:].isfinite().all())
    _check(bc, held[:1], lens[:1], q, k, v, out, fill=None)
    assert not bool(rows[:2].isnan().any())
    # a page with the scale NaN: its place's head reads as NaN, the others as before
    before = out.clone()
    bc.k_scale[0, int(bc.table[0, 1]), 1] = float("nan")
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    assert bool(out[:a1, 4:].isnan().all())
    assert torch.equal(out[:a1, :4].view(torch.int16), before[:a1, :4].view(torch.int16))
    assert torch.equal(out[a1:].view(torch.int16), before[a1:].view(torch.int16))
    bc.v_scale[0, int(bc.table[2, 0]), 0] = float("nan")
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    assert bool(out[a2:, :4].isnan().all()) and not bool(out[a2:, 4:].isnan().any())


@pytest.mark.parametrize("lens", [[5, 3], [90, 40], [300, 260]])
def test_logits_and_scales_of_every_size(lens):
    """Values of blocks 2^40 apart, sharp logits, queries from 2^-133 to 2^100 beside keys that
    give ordinary logits."""
    import torch
    held = [700, 260]
    bc = _cache(held, 8, 2, sum(lens), seed=21, extra=400, fill=0.0)
    for s in range(2):
        pages = bc.table[s, :held[s] // N].long()
        f = 2.0 ** (20 * (torch.arange(len(pages), device="cuda") % 5 - 2).float())
        bc.v_scale[0, pages] *= f[:, None]
    _run(bc, held, lens, seed=22)
    _run(bc, held, lens, seed=23, scale=40.0, loose=4.0)    # (logits to 500: 2^-24 x 128 x 4000 / 11 = 2^-8.4, twice)
    for e in (100, 60, -60, -100):
        b = _cache(held, 8, 2, sum(lens), seed=24, extra=400, fill=0.0)
        b.k_scale *= 2.0 ** -e
        b.k_tail.copy_((b.k_tail.float() * 2.0 ** -e).bfloat16())
        q, k, v = _rows(sum(lens), 8, 2, seed=25)
        q, k = (q.float() * 2.0 ** e).bfloat16(), (k.float() * 2.0 ** -e).bfloat16()
        out = torch.full_like(q, 7.0)
        b.attend_chunk(0, q, k, v, _cu(lens), out)
        _check(b, held, lens, q, k, v, out)
    # queries of bf16's smallest values, of zeros
    b = _cache(held, 8, 2, sum(lens), seed=26, extra=400, fill=0.0)
    q, k, v = _rows(sum(lens), 8, 2, seed=27)
    for e in (-133, -130):
        q = (torch.randint(-3, 4, q.shape, device="cuda").double() * 2.0 ** e).float().bfloat16()
        b.k_scale.copy_(torch.full_like(b.k_scale, 2.0 ** 120))
        b.k_tail.fill_(2.0 ** 120)
        out = torch.full_like(q, 7.0)
        b.attend_chunk(0, q, (k.float() * 2.0 ** 100).bfloat16(), v, _cu(lens), out)
        _check(b, held, lens, q, (k.float() * 2.0 ** 100).bfloat16(), v, out)
    q.zero_()
    b.attend_chunk(0, q, k, v, _cu(lens), out)
    _check(b, held, lens, q, k, v, out)


@pytest.mark.parametrize("lens", [[5, 3], [90, 40], [300, 260]])
def test_value_scales_far_apart(lens):
    """Values of a block 2^79 to 2^100 smaller than those of the next, blocks of zeros (with the
    smallest scale, or a scale of zero): their keys weigh in a row's sum as all others do."""
    import torch
    held = [700, 260]
    bc = _cache(held, 8, 2, sum(lens), seed=50, extra=400, fill=0.0)
    small = [1.0, 2.0 ** -79, 2.0 ** -81, 0.0, 2.0 ** -100]
    for s in range(2):
        pages = bc.table[s, :held[s] // N].long()
        for i, p in enumerate(pages.tolist()):
            bc.v_scale[0, p] *= small[i % 5]
    _run(bc, held, lens, seed=51)
    _run(bc, held, lens, seed=52, scale=8.0)
    bc.v_scale.fill_(2.0 ** -100)
    bc.v_codes.zero_()
    _run(bc, held, lens, seed=53)
    bc = _cache(held, 8, 2, sum(lens), seed=54, extra=400, fill=0.0)
    bc.v_scale *= 2.0 ** -90                  # all of a place's values
    bc.v_tail.copy_(bc.v_tail.float() * 2.0 ** -90)
    q, k, v = _rows(sum(lens), 8, 2, seed=55)
    v = (v.float() * 2.0 ** -90).bfloat16()
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, _cu(lens), out)
    _check(bc, held, lens, q, k, v, out)


def test_softmax_scale():
    import paper_2608_05326_amd as qv
    import torch
    held, lens = [200, 77], [30, 4]
    base = _cache(held, 4, 2, 34, seed=28)
    for scale in (0.3, 2.0 ** -64, 2.0 ** -10):
        bc = qv.BlockCache(qv.BlockConfig(2, 4, 2, base.cfg.max_context, num_pages=base.num_pages, softmax_scale=scale,
                                          chunk_tokens=34))
        for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "lens"):
            setattr(bc, name, getattr(base, name))
        q, k, v = _rows(34, 4, 2, seed=30)
        out = torch.full_like(q, 7.0)
        bc.attend_chunk(0, q, k, v, _cu(lens), out)
        _check(bc, held, lens, q, k, v, out, scale=scale)


def test_bitwise_repeatable_and_captured():
    """Replays while lengths, tables and chunks move, beside eager steps of another cache."""
    import torch
    held, T = [0, 700, 64, 3000], 60
    bc = _cache(held, 8, 2, T, seed=31, extra=200, fill=0.0)
    other = _cache(held, 8, 2, T, seed=31, extra=200, fill=0.0)
    q, k, v = _rows(T, 8, 2, seed=32)
    cu = _cu([30, 3, 20, 7])
    out, want = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bc.attend_chunk(0, q, k, v, cu, out)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        bc.attend_chunk(0, q, k, v, cu, out)
    rng = np.random.default_rng(1)
    for i in range(6):
        n = rng.multinomial(T, [0.25] * 4)
        cu.copy_(_cu(n))
        lens = torch.tensor([int(rng.integers(-1, h + 1)) for h in held], dtype=torch.int32)
        bc.lens, other.lens = lens, lens
        q.copy_(_bf16(T, 8, D, seed=50 + i))
        out.fill_(7.0)
        want.fill_(7.0)
        g.replay()
        other.attend_chunk(0, q, k, v, cu, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        _check(bc, lens.tolist(), n.tolist(), q, k, v, out)


def test_two_calls_at_once():
    """Caches of their own on two streams."""
    import torch
    held, lens = [3000, 100, 2000], [40, 4, 300]
    a, b = (_cache(held, 8, 2, sum(lens), seed=s, extra=400, fill=0.0) for s in (33, 34))
    q, k, v = _rows(sum(lens), 8, 2, seed=35)
    cu = _cu(lens)
    want = [torch.zeros_like(q) for _ in range(2)]
    for x, w in zip((a, b), want):
        x.attend_chunk(0, q, k, v, cu, w)
    torch.cuda.synchronize()
    outs = [[torch.zeros_like(q) for _ in range(8)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(8):
        for x, st, o in zip((a, b), streams, outs):
            with torch.cuda.stream(st):
                x.attend_chunk(0, q, k, v, cu, o[i])
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, x) for x in o)


def test_pages_and_rows_past_2_to_the_31():
    import paper_2608_05326_amd as qv
    import torch
    hkv, T, st = 4, 600, 1 << 22
    pages = (1 << 31) // (hkv * N * D) + 40
    bc = qv.BlockCache(qv.BlockConfig(1, 4, hkv, 2000, num_pages=pages, chunk_tokens=T))
    bc.table = torch.arange(pages - 32, pages, dtype=torch.int32)[None]
    k0, v0 = (_bf16(1000, hkv, D, seed=s).cuda() for s in (36, 37))
    bc.store(0, k0, v0, _cu([1000]))
    bc.lens = torch.tensor([1000], dtype=torch.int32)
    buf = torch.empty((T - 1) * st + 4 * hkv * D, dtype=torch.bfloat16, device="cuda")
    q, k, v, out = (buf.as_strided((T, hkv, D), (st, D, 1), i * hkv * D) for i in range(4))
    for x, y in zip((q, k, v), _rows(T, hkv, hkv, seed=38)):
        x.copy_(y)
    bc.attend_chunk(0, q, k, v, _cu([T]), out)
    _check(bc, [1000], [T], q, k, v, out)


def test_a_prompt_in_pieces_and_drafted_tokens():
    """rotate, attend_chunk, append and advance as a program uses them: prompts in pieces of any
    size beside each other, then drafted tokens of which some are kept; two layers."""
    import paper_2608_05326_amd as qv
    import torch
    hq, hkv, B, layers = 8, 2, 4, 2
    prompt = [500, 130, 64, 1]
    bc = qv.BlockCache(qv.BlockConfig(B, hq, hkv, 700, num_layers=layers, chunk_tokens=400))
    r = qv.Rotary(base=500000.0, sections=(16, 24, 24))
    bc.lens = torch.zeros(B, dtype=torch.int32)
    rng = np.random.default_rng(3)
    at, step = [0] * B, 0
    kept = [[[], []] for _ in range(layers)]          # rotated keys and values by layer, place 0's
    while step < 16:
        drafted = all(a >= p for a, p in zip(at, prompt))
        n = [int(rng.integers(1, 7)) if drafted else min(p - a, int(rng.integers(0, 120))) for a, p in zip(at, prompt)]
        take = [int(rng.integers(0, x + 1)) if drafted else x for x in n]
        T, cu = sum(n), _cu(n)
        counts = torch.tensor(take, dtype=torch.int32).cuda() if drafted else None
        pos = torch.cat([torch.arange(a, a + x) for a, x in zip(at, n)]).to(torch.int32).cuda()
        pos = torch.stack([pos, pos // 32, pos % 32], 1)
        for layer in range(layers):
            q, k, v = _rows(T, hq, hkv, seed=100 * step + layer)
            qr, kr = qv.rotate(q, k, pos, r)
            out = torch.full_like(q, 7.0)
            bc.attend_chunk(layer, qr, kr, v, cu, out)
            _check(bc, at, n, qr, kr, v, out, layer=layer)
            bc.append(layer, k, v, cu, r, pos, counts)
            kept[layer][0].append(kr[:take[0]])
            kept[layer][1].append(v[:take[0]])
        bc.advance(cu, counts)
        at = [a + x for a, x in zip(at, take)]
        assert bc.lens.tolist() == at
        step += 1
    assert all(a >= p for a, p in zip(at, prompt))
    # what the cache holds of place 0: bf16 in the open block, half a step of its scale elsewhere
    for layer in range(layers):
        for got, want in zip(zip(*[_held(bc, 0, h, at[0], layer)[:2] for h in range(hkv)]), kept[layer]):
            got, want = torch.stack(got, 1), torch.cat(want).double()
            n = at[0] // N * N
            assert torch.equal(got[n:], want[n:])
            step_size = want[:n].view(-1, N, hkv, D).abs().amax(dim=(1, 3)) / 127
            err = (got[:n] - want[:n]).abs().view(-1, N, hkv, D).amax(dim=(1, 3))
            assert bool((err <= step_size * (0.5 + 2.0 ** -16)).all())


def test_the_cache_is_only_read():
    import torch
    held, lens = [500, 64], [70, 3]
    bc = _cache(held, 8, 2, 73, seed=39)
    names = ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "lens")
    before = {n: getattr(bc, n).clone() for n in names}
    q, k, v = _rows(73, 8, 2, seed=40)
    rows = [x.clone() for x in (q, k, v)]
    bc.attend_chunk(0, q, k, v, _cu(lens), torch.empty_like(q))
    for n in names:
        a, b = before[n].flatten(), getattr(bc, n).flatten()
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), n
    assert all(torch.equal(x, y) for x, y in zip(rows, (q, k, v)))


def test_refusals():
    import torch
    bc = _cache([100, 5], 8, 2, 50, seed=41)
    q, k, v = _rows(50, 8, 2, seed=42)
    cu, out = _cu([40, 10]), torch.empty_like(q)
    for args in ((q[:49], k, v, cu, out), (q, k[:, :1], v, cu, out), (q, k, v.float(), cu, out),
                 (q, k, v, cu[:2], out), (q, k, v, cu.long(), out), (q, k, v, cu, out[:, :4]),
                 (q.cpu(), k, v, cu, out), (q[..., :64], k, v, cu, out)):
        with pytest.raises(ValueError):
            bc.attend_chunk(0, *args)
    with pytest.raises(ValueError):
        bc.attend_chunk(1, q, k, v, cu, out)
    big = torch.cat([q, q])
    with pytest.raises(ValueError, match="chunk_tokens"):
        bc.attend_chunk(0, big, torch.cat([k, k]), torch.cat([v, v]), cu, big.clone())
    bc.attend_chunk(0, q[:0], k[:0], v[:0], cu, out[:0])
    _check(bc, [100, 5], [40, 10], q, k, v, _once(bc, q, k, v, cu))


def _once(bc, q, k, v, cu):
    import torch
    out = torch.full_like(q, 7.0)
    bc.attend_chunk(0, q, k, v, cu, out)
    return out
