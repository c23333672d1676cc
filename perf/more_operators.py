"""Chunks of new tokens over the 8-bit block cache, as cases that can be timed and compared.

Three operators, each as a serving program calls it through the Python binding:

  rotate  rotary positions with one or several axes on the queries and keys of a projection
  append  new tokens behind the tokens of every sequence of a block cache (64-token blocks,
          int8 codes with a scale for each block and KV head, the open block in bf16), with
          the keys rotated on the way or as they are; the blocks that the new tokens
          complete are returned as the values they stand for
  chunk   attention of a chunk of new tokens for every sequence over the block cache and the
          chunk itself (a piece of a prompt, drafted tokens to verify, or one token)

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits
(64 for angles and for the decision of a code); with ``own`` true it calls the library.

A cache is plain tensors: codes [pages, H_kv, 64, d] (keys) and [pages, H_kv, d, 64]
(values) int8, scales [pages, H_kv] fp32, open blocks [B, H_kv, 64, d] bf16, a page table
[B, blocks] and lengths [B] int32.  A page is written by one sequence at a time.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
BLOCK = 64
MIN_SCALE = 2.0 ** -100
BASE = 500000.0


# ------------------------------------------------------------------- cases
def listed():
    return [
        # --- rotate ---
        # one new token for each of 32 sequences: the smallest call, where latency counts
        dict(name="rotate_decode_b32", kind="rotate", hq=32, hkv=8, tokens=32, sections="64", fused=True),
        # an image and its text in a 70B-shaped layer: time, height and width
        dict(name="rotate_image_70b", kind="rotate", hq=64, hkv=8, tokens=4999, sections="16,24,24", fused=True),
        # a whole 32K prompt of an 8B-shaped layer
        dict(name="rotate_8b_32k", kind="rotate", hq=32, hkv=8, tokens=32768, sections="64", fused=False),
        # --- append ---
        # a few accepted tokens of eight sequences, some of which complete a block
        dict(name="append_drafted_b8", kind="append", hkv=8, held="2067,1000,63,0,8127,300,16380,640",
             lens="5,1,1,4,1,3,4,2", sections="64", rotate=False, fused=True),
        # a document's kept keys (before any rotation) and values behind four short instructions
        dict(name="append_document", kind="append", hkv=8, held="128,47,960,0", lens="2500,1041,4096,4133",
             sections="64", rotate=True, fused=False),
        # pieces of 16 prompts in a large batch, with image positions
        dict(name="append_pieces_b16", kind="append", hkv=8,
             held="30016,64,1000,0,8192,20000,4096,12,5000,640,100,63,2048,16384,7777,1",
             lens="2048,1999,24,513,4096,96,2047,1,2040,700,1820,1,2000,1024,31,63",
             sections="16,24,24", rotate=True, fused=True),
        # --- chunk ---
        # five drafted tokens of one 2K sequence on a small model: the smallest step
        dict(name="chunk_drafted_2k", kind="chunk", hq=8, hkv=8, held="2067", lens="5", fused=False),
        # drafted tokens of 32 sequences of a 70B-shaped layer, some places empty or idle
        dict(name="chunk_drafted_70b_b32", kind="chunk", hq=64, hkv=8,
             held="131072,0,63,64,1000,-1,20000,32768,5,4095,16000,127,9000,40000,2067,300,"
                  "-1,12345,65535,777,8192,6400,1,30000,25000,11111,2222,33333,4444,5555,-1,18000",
             lens="4,5,4,1,4,0,4,4,8,4,4,4,0,4,3,4,0,4,2,4,4,4,7,4,4,1,4,4,6,4,0,4", fused=True),
        # 512 tokens of a prompt whose first 32K are held: the ordinary piece of a long prompt
        dict(name="chunk_8b_512_at_32k", kind="chunk", hq=32, hkv=8, held="32768", lens="512", fused=True),
        # a piece of one prompt beside fifteen sequences that decode
        dict(name="chunk_mixed_b16", kind="chunk", hq=32, hkv=8,
             held="14001,32768,30001,16383,24576,32700,8191,20480,29999,5000,1000,63,27000,12345,18000,9000",
             lens="2048,1,1,1,1,1,1,1,1,1,1,1,1,1,1,1", fused=True),
        # pieces of four prompts with seven query heads to a KV head
        dict(name="chunk_pieces_gqa7", kind="chunk", hq=28, hkv=4, held="0,8192,3000,20011", lens="1777,1024,333,2048",
             fused=False),
        # a large piece of a long prompt in a 70B-shaped layer
        dict(name="chunk_70b_4k_at_60k", kind="chunk", hq=64, hkv=8, held="61440", lens="4096", fused=False),
    ]


_HEADS = [(8, 8), (32, 8), (64, 8), (16, 2), (28, 4)]
_SECTIONS = ["64", "16,24,24", "20,22,22", "32,32"]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges of listed(), without a name."""
    kind = rng.choice(["rotate", "append", "chunk", "chunk"])
    hq, hkv = rng.choice(_HEADS)
    if kind == "rotate":
        return dict(kind=kind, hq=hq, hkv=hkv, tokens=_log_int(rng, 1, 32768 * 40 // max(hq + hkv, 40)),
                    sections=rng.choice(_SECTIONS), fused=rng.random() < 0.5)
    n = _log_int(rng, 1, 32)
    held, lens = [], []
    if kind == "append":
        room = 20000 * 8 // hkv
        for _ in range(n):
            a, t = rng.choice([0, _log_int(rng, 1, 32768)]), min(_log_int(rng, 1, 8192), room)
            if a % BLOCK and a % BLOCK + t >= BLOCK:
                # a pass can be repeated: the open block that is completed is not written over
                t += -(a + t) % BLOCK
            if t > room:
                break
            held.append(a)
            lens.append(t)
            room -= t
        if not lens:
            held, lens = [0], [1]
        return dict(kind=kind, hkv=hkv, held=",".join(map(str, held)), lens=",".join(map(str, lens)),
                    sections=rng.choice(_SECTIONS), rotate=rng.random() < 0.5, fused=rng.random() < 0.5)
    room, keys = 4096.0 * 63488 * 64 / hq, 470000 * 8 // hkv
    most = rng.choice([8, 4096])      # drafted tokens, or pieces of prompts
    for _ in range(n):
        if n > 1 and rng.random() < 0.1:
            held.append(-1)
            lens.append(0)
            continue
        a = min(rng.choice([0, _log_int(rng, 1, 131072), _log_int(rng, 1, 131072)]), keys)
        t = min(_log_int(rng, 1, most), int(room / (a + 4096)))
        if t < 1:
            break
        held.append(a)
        lens.append(t)
        room -= t * (a + t)
        keys -= a
    if not sum(lens):
        held, lens = [100], [3]
    return dict(kind=kind, hq=hq, hkv=hkv, held=",".join(map(str, held)), lens=",".join(map(str, lens)),
                fused=hq > 8 and rng.random() < 0.5)


def _ints(case, name):
    return [int(x) for x in case[name].split(",")]


def work(case):
    hkv = case["hkv"]
    if case["kind"] == "rotate":
        n, axes = case["tokens"], len(_ints(case, "sections"))
        rows = n * (case["hq"] + hkv)
        return {"bytes": rows * D * 4 + n * axes * 4, "flops": rows * D * 3}
    held, lens = _ints(case, "held"), _ints(case, "lens")
    if case["kind"] == "append":
        total = sum(lens)
        whole = sum((a + t) // BLOCK - a // BLOCK for a, t in zip(held, lens))
        opened = sum(a % BLOCK for a, t in zip(held, lens) if a % BLOCK + t >= BLOCK)    # read back, in bf16
        left = sum((a + t) % BLOCK if a % BLOCK + t >= BLOCK else t for a, t in zip(held, lens))
        positions = total * len(_ints(case, "sections")) * 4 if case["rotate"] else 0
        # codes are written, and read again for the values that come out in bf16
        return {"bytes": hkv * (total * 4 * D + opened * 4 * D + left * 4 * D + whole * (BLOCK * D * 8 + 16)) + positions,
                "flops": hkv * (total * 4 * D + (total * 3 * D if case["rotate"] else 0))}
    hq = case["hq"]
    live = [(a, t) for a, t in zip(held, lens) if a >= 0 and t > 0]
    cache = sum(a // BLOCK * (BLOCK * 2 * D + 8) + a % BLOCK * 4 * D for a, _ in live) * hkv
    return {"bytes": cache + sum(lens) * (2 * hq + 2 * hkv) * D * 2,
            "flops": 4 * D * hq * sum(t * a + t * (t + 1) // 2 for a, t in live)}


# ------------------------------------------------------------------ inputs
def _cu(lens):
    cu = [0]
    for t in lens:
        cu.append(cu[-1] + t)
    return cu


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _frequencies():
    """Radians a position, of the 64 pairs (i, i + 64)."""
    return [BASE ** (-2.0 * i / D) for i in range(D // 2)]


def _axis_of_pairs(case):
    return [a for a, n in enumerate(_ints(case, "sections")) for _ in range(n)]


def _positions(case, g, starts, lens):
    """int32 [tokens, axes]: text counts on, a picture of 32 columns has rows and columns."""
    axes, total = len(_ints(case, "sections")), sum(lens)
    at = torch.cat([torch.arange(a, a + t, device="cuda") for a, t in zip(starts, lens)])
    if axes == 1:
        return at[:, None].to(torch.int32).contiguous()
    first = torch.repeat_interleave(torch.tensor(starts, device="cuda"), torch.tensor(lens, device="cuda"))
    i = at - first
    text = torch.rand(total, generator=g, device="cuda") < 0.25
    grid = torch.stack([first + i // 1024, first + i // 32 % 32, first + i % 32], dim=1)[:, 3 - axes:]
    return torch.where(text[:, None], at[:, None], grid).to(torch.int32).contiguous()


def _packed_rows(case, total, hq, g):
    """q, k, v [tokens, heads, d] bf16: normal keys and values, queries drawn towards one
    direction per KV head that some keys share (heads attend to a few tokens sharply)."""
    hkv = case["hkv"]
    if case["fused"]:
        buf = _normal(g, total, hq + 2 * hkv, D).bfloat16()
        q, k, v = buf[:, :hq], buf[:, hq:hq + hkv], buf[:, hq + hkv:]
    else:
        q, k, v = (_normal(g, total, h, D).bfloat16() for h in (hq, hkv, hkv))
    u = _normal(g, hkv, D)
    u /= u.norm(dim=1, keepdim=True)
    if hq:
        q += (3.0 * u).repeat_interleave(hq // hkv, dim=0).bfloat16()
    mark = (torch.rand(total, hkv, 1, generator=g, device="cuda") < 0.02).float()
    k += (mark * (12.0 * u)).bfloat16()
    return q, k, v


def _cache_tensors(case, g, held, lens, fill):
    """The tensors of a cache whose sequences hold `held` tokens and get `lens` more, pages
    in no order; the pages of the blocks that are completed are the pool's last `fresh`."""
    hkv, n = case["hkv"], len(held)
    n_cols = max(max(a, 0) + t for a, t in zip(held, lens)) // BLOCK + 1
    full = [max(a, 0) // BLOCK for a in held]
    done = [(max(a, 0) + t) // BLOCK - f for a, t, f in zip(held, lens, full)]
    fresh = sum(done)
    # the pages that are held; where the cache is not read they are named and not kept
    n_old = sum(full) + 3 if fill else 3
    n_pages = n_old + fresh
    old = torch.randperm(n_old, generator=g, device="cuda").to(torch.int32)
    new = (n_old + torch.randperm(fresh, generator=g, device="cuda")).to(torch.int32)
    table = torch.full((n, n_cols), -1, dtype=torch.int32, device="cuda")
    at_old = at_new = 0
    for s, (f, d) in enumerate(zip(full, done)):
        if fill:
            table[s, :f] = old[at_old:at_old + f]
        table[s, f:f + d] = new[at_new:at_new + d]
        at_old, at_new = at_old + f, at_new + d
    c = dict(table=table, lens=torch.tensor(held, dtype=torch.int32, device="cuda"), fresh=(n_old, n_pages))
    for name, shape in (("k_codes", (n_pages, hkv, BLOCK, D)), ("v_codes", (n_pages, hkv, D, BLOCK))):
        c[name] = torch.zeros(shape, dtype=torch.int8, device="cuda")
        sc = torch.full((n_pages, hkv), MIN_SCALE, dtype=torch.float32, device="cuda")
        if fill:
            for a in range(0, n_old, 1024):
                b = min(a + 1024, n_old)
                x = _normal(g, *((b - a,) + shape[1:]))
                s = x.abs().amax(dim=(2, 3)) / 127.0
                sc[a:b] = s
                c[name][a:b] = torch.round(x / s[:, :, None, None]).clamp_(-127, 127).to(torch.int8)
        c[name[0] + "_scale"] = sc
    for name in ("k_tail", "v_tail"):
        c[name] = _normal(g, n, hkv, BLOCK, D).bfloat16()
    return c


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    st = dict(case=case)
    if case["kind"] == "rotate":
        n = case["tokens"]
        st["q"], st["k"], _ = _packed_rows(case, n, case["hq"], g)
        # 32 decoding sequences are anywhere in their contexts, a prompt's tokens in order
        starts = torch.randint(0, 131072, (n,), generator=g, device="cuda").tolist() if n <= 64 else \
            torch.randint(0, 65536, (1,), generator=g, device="cuda").tolist()
        st["positions"] = _positions(case, g, starts, [1] * n if n <= 64 else [n])
        st["q_out"], st["k_out"] = (torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda")
                                    for x in (st["q"], st["k"]))
        return st
    held, lens = _ints(case, "held"), _ints(case, "lens")
    st["held"], st["lens"], st["cu_host"] = held, lens, _cu(lens)
    st["cu"] = torch.tensor(st["cu_host"], dtype=torch.int32, device="cuda")
    st["q"], st["k"], st["v"] = _packed_rows(case, sum(lens), case.get("hq", 0), g)
    st["cache"] = c = _cache_tensors(case, g, held, lens, fill=case["kind"] == "chunk")
    if case["kind"] == "chunk":
        st["out"] = torch.zeros(st["q"].shape, dtype=torch.bfloat16, device="cuda")
    else:
        st["positions"] = _positions(case, g, held, lens)
        a, b = c["fresh"]
        st["k_done"], st["v_done"] = (torch.zeros((b - a,) + c[x].shape[1:], dtype=torch.bfloat16, device="cuda")
                                      for x in ("k_codes", "v_codes"))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        import paper_2608_05326_amd as qv
        if "sections" in case:
            st["rotary"] = qv.Rotary(base=BASE, sections=_ints(case, "sections"))
        if "cache" in st:
            c, hkv = st["cache"], case["hkv"]
            bc = qv.BlockCache(qv.BlockConfig(
                batch=len(st["lens"]), num_q_heads=case.get("hq", hkv), num_kv_heads=hkv,
                max_context=c["table"].shape[1] * BLOCK, num_pages=c["k_codes"].shape[0],
                chunk_tokens=sum(st["lens"]) if case["kind"] == "chunk" else 0))
            for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail"):
                getattr(bc, name)[0].copy_(c[name])
                c[name] = getattr(bc, name)[0]
            bc.table.copy_(c["table"])
            bc.lens.copy_(c["lens"])
            st["handle"] = bc
    return st


# ---------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_rotate(st):
    import paper_2608_05326_amd as qv
    return qv.rotate(st["q"], st["k"], st["positions"], st["rotary"], st["q_out"], st["k_out"])


def _own_append(st):
    if st["case"]["rotate"]:
        st["handle"].append(0, st["k"], st["v"], st["cu"], st["rotary"], st["positions"])
    else:
        st["handle"].append(0, st["k"], st["v"], st["cu"])
    return _append_outputs(st)


def _append_outputs(st):
    """The open blocks, and the values of the blocks just completed."""
    c = st["cache"]
    a, b = c["fresh"]
    if a == b:
        return c["k_tail"], c["v_tail"]
    return (c["k_tail"], c["v_tail"],
            torch.mul(c["k_codes"][a:b], c["k_scale"][a:b, :, None, None], out=st["k_done"]),
            torch.mul(c["v_codes"][a:b], c["v_scale"][a:b, :, None, None], out=st["v_done"]))


def _own_chunk(st):
    st["handle"].attend_chunk(0, st["q"], st["k"], st["v"], st["cu"], st["out"])
    return st["out"]


def _rotated(x, positions, case):
    """x [tokens, heads, d] in 32 bits, angles in 64."""
    axis = torch.tensor(_axis_of_pairs(case), device="cuda")
    f = torch.tensor(_frequencies(), dtype=torch.float64, device="cuda")
    t = positions[:, axis].double() * f
    cos, sin = torch.cos(t).float()[:, None], torch.sin(t).float()[:, None]
    x = x.float()
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_rotate(st):
    st["q_out"].copy_(_rotated(st["q"], st["positions"], st["case"]))
    st["k_out"].copy_(_rotated(st["k"], st["positions"], st["case"]))
    return st["q_out"], st["k_out"]


def _quantize(x):
    """Blocks [..., 64, d] -> int8 codes, fp32 scales [...]: half-step decisions in 64 bits."""
    s = (x.float().abs().amax(dim=(-2, -1)).double() / 127.0).float().clamp_min(MIN_SCALE)
    return torch.round(x.double() / s.double()[..., None, None]).to(torch.int8), s


def _plain_append(st):
    c, held, cu = st["cache"], st["held"], st["cu_host"]
    k, v = st["k"], st["v"]
    if st["case"]["rotate"]:
        k = _rotated(k, st["positions"], st["case"]).bfloat16()
    for s, (a, b) in enumerate(zip(cu, cu[1:])):
        r, first = held[s] % BLOCK, held[s] // BLOCK
        n = (r + b - a) // BLOCK
        # the open block's rows and the new ones, [H_kv, rows, d]
        kv = [torch.cat([c[t][s, :, :r], x[a:b].transpose(0, 1)], dim=1) for t, x in (("k_tail", k), ("v_tail", v))]
        if n:
            pages = c["table"][s, first:first + n].long()
            blocks = [x[:, :n * BLOCK].reshape(-1, n, BLOCK, D).transpose(0, 1) for x in kv]
            c["k_codes"][pages], c["k_scale"][pages] = _quantize(blocks[0])
            codes, c["v_scale"][pages] = _quantize(blocks[1])
            c["v_codes"][pages] = codes.transpose(-1, -2)
        for t, x in zip(("k_tail", "v_tail"), kv):
            c[t][s, :, :r + b - a - n * BLOCK] = x[:, n * BLOCK:]
    return _append_outputs(st)


def _sequence(c, s, t):
    """fp32 keys and values [H_kv, t, d] of sequence s."""
    n = t // BLOCK
    p = c["table"][s, :n].long()
    k = (c["k_codes"][p].float() * c["k_scale"][p][:, :, None, None]).transpose(0, 1)
    v = (c["v_codes"][p].float() * c["v_scale"][p][:, :, None, None]).permute(1, 0, 3, 2)
    hkv = k.shape[0]
    return [torch.cat([x.reshape(hkv, n * BLOCK, D), c[tail][s, :, :t - n * BLOCK].float()], dim=1)
            for x, tail in ((k, "k_tail"), (v, "v_tail"))]


def _plain_chunk(st):
    c, hq, hkv = st["cache"], st["case"]["hq"], st["case"]["hkv"]
    g, rows = hq // hkv, 1024
    for s, (a, b) in enumerate(zip(st["cu_host"], st["cu_host"][1:])):
        if a == b:
            continue
        t = st["held"][s]
        k, v = _sequence(c, s, t)
        k = torch.cat([k, st["k"][a:b].float().transpose(0, 1)], dim=1).transpose(1, 2).contiguous()   # [hkv, d, keys]
        v = torch.cat([v, st["v"][a:b].float().transpose(0, 1)], dim=1)
        q = st["q"][a:b].float().view(b - a, hkv, g, D)
        pos = torch.arange(t + b - a, device="cuda")
        for r in range(0, b - a, rows):
            e = min(r + rows, b - a)
            qr = q[r:e].permute(1, 2, 0, 3).reshape(hkv, g * (e - r), D)
            w = (qr @ k[:, :, :t + e].contiguous()).view(hkv, g, e - r, t + e) / math.sqrt(D)
            w.masked_fill_(pos[None, :t + e] > pos[t + r:t + e, None], -math.inf)
            w = torch.exp(w - w.amax(dim=-1, keepdim=True))
            w = w / w.sum(dim=-1, keepdim=True)
            o = w.view(hkv, g * (e - r), t + e) @ v[:, :t + e].contiguous()
            st["out"][a + r:a + e] = o.view(hkv, g, e - r, D).permute(2, 0, 1, 3).reshape(e - r, hq, D)
    return st["out"]


_PLAIN = dict(rotate=_plain_rotate, append=_plain_append, chunk=_plain_chunk)
_OWN = dict(rotate=_own_rotate, append=_own_append, chunk=_own_chunk)


# --------------------------------------------------- results in 64 bits
def _exact_rotation(x, positions, case):
    """x [tokens, heads, d] -> float64: every pair times a complex number of length one."""
    z = torch.complex(x[..., :D // 2].double(), x[..., D // 2:].double())
    turn = torch.empty(x.shape[0], D // 2, dtype=torch.float64, device="cuda")
    at = 0
    for axis, n in enumerate(_ints(case, "sections")):
        for i in range(at, at + n):
            turn[:, i] = positions[:, axis].double() * BASE ** (-i / (D / 2))
        at += n
    z = z * torch.polar(torch.ones_like(turn), turn)[:, None]
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_values(rows):
    """[64, d] of one block and head -> the float64 values that its codes stand for."""
    x = rows.double()
    scale = (x.abs().amax() / 127.0).float().clamp_min(MIN_SCALE).double()
    return torch.round(x / scale) * scale


def _exact_append(case, st):
    c, hkv = st["cache"], case["hkv"]
    k, v = st["k"], st["v"]
    if case["rotate"]:   # what is kept is the rotated key in its type
        k = _exact_rotation(k, st["positions"], case).to(torch.bfloat16)
    tails = [c["k_tail"].double().clone(), c["v_tail"].double().clone()]
    first, last = c["fresh"]
    done = [torch.zeros(last - first, hkv, *shape, dtype=torch.float64, device="cuda")
            for shape in ((BLOCK, D), (D, BLOCK))]
    for s, (a, b) in enumerate(zip(st["cu_host"], st["cu_host"][1:])):
        begin = st["held"][s]
        for j, (x, tail) in enumerate(((k, c["k_tail"]), (v, c["v_tail"]))):
            for blk in range(begin // BLOCK, (begin + b - a - 1) // BLOCK + 1):
                # the block's rows that are there: held ones and new ones
                lo, hi = max(blk * BLOCK, begin), min(blk * BLOCK + BLOCK, begin + b - a)
                rows = torch.cat([tail[s, :, :lo - blk * BLOCK], x[a + lo - begin:a + hi - begin].transpose(0, 1)],
                                 dim=1)
                if hi - blk * BLOCK < BLOCK:
                    tails[j][s, :, :rows.shape[1]] = rows.double()
                    continue
                page = int(c["table"][s, blk]) - first
                for h in range(hkv):
                    y = _exact_values(rows[h])
                    done[j][page, h] = y.t() if j else y
    return tuple(tails) if first == last else tuple(tails + done)


def _exact_chunk(case, st):
    c, hq, hkv = st["cache"], case["hq"], case["hkv"]
    group = hq // hkv
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, (a, b) in enumerate(zip(st["cu_host"], st["cu_host"][1:])):
        if a == b:
            continue
        t = st["held"][s]
        n = t // BLOCK
        pages = c["table"][s, :n].long()
        for h in range(hkv):
            kv = []
            for name in "kv":
                codes = c[name + "_codes"][pages, h].double()
                if name == "v":
                    codes = codes.transpose(1, 2)
                whole = (codes * c[name + "_scale"][pages, h].double().view(n, 1, 1)).reshape(n * BLOCK, D)
                kv.append(torch.cat([whole, c[name + "_tail"][s, h, :t - n * BLOCK].double(),
                                     st[name][a:b, h].double()]))
            keys = kv[0].t().contiguous()
            for head in range(h * group, h * group + group):
                for r in range(a, b, 4096):
                    e = min(r + 4096, b)
                    logits = st["q"][r:e, head].double() @ keys[:, :t + e - a].contiguous() * D ** -0.5
                    seen = torch.arange(t + e - a, device="cuda")[None] <= torch.arange(t + r - a, t + e - a,
                                                                                       device="cuda")[:, None]
                    logits = torch.where(seen, logits, -math.inf)
                    out[r:e, head] = torch.softmax(logits, dim=1) @ kv[1][:t + e - a]
    return out


def exact(case, seed):
    """What run returns for these inputs, in float64 from the definitions."""
    st = _inputs(case, seed)
    if case["kind"] == "rotate":
        return tuple(_exact_rotation(st[x], st["positions"], case) for x in "qk")
    if case["kind"] == "append":
        return _exact_append(case, st)
    return _exact_chunk(case, st)
