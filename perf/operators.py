"""Causal attention over packed prompts and the 8-bit block cache, as cases that can be
timed and compared.

Four operators, each as a serving program calls it through the Python binding:

  prompt  attention of whole prompts, packed one behind the other: every token over the
          tokens of its own prompt up to itself, grouped query heads
  store   prompts into the 8-bit block cache (64-token blocks, a scale for each block and
          KV head, the open block in bf16); the cache is read back, so the outputs are the
          values it stands for
  fetch   sequences of the block cache back into packed bf16 keys and values
  attend  one decode token for every sequence of a block cache: append, attend, and close
          the blocks that the token fills

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits
(64 for the decision of a code); with ``own`` true it calls the library.

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


# ------------------------------------------------------------------- cases
def listed():
    return [
        # --- prompts ---
        # short requests of a chat service, admitted together: eight prompts of 1 to 214
        # tokens, queries, keys and values as slices of one projection's output
        dict(name="prompt_short", kind="prompt", hq=32, hkv=8, lens="1,37,214,64,9,128,65,150", fused=True),
        # one 2K prompt of a small model without head groups
        dict(name="prompt_2k", kind="prompt", hq=8, hkv=8, lens="2067", fused=False),
        # a 70B-shaped layer, prompts of very different lengths in one batch
        dict(name="prompt_70b_packed", kind="prompt", hq=64, hkv=8, lens="4096,1000,7777,33,2500,513", fused=True),
        # an 8B-shaped layer's whole 32K prompt: the longest prompt of the benchmark's model
        dict(name="prompt_8b_32k", kind="prompt", hq=32, hkv=8, lens="32768", fused=False),
        # --- store ---
        # the short requests' prompts into the cache
        dict(name="store_short", kind="store", hkv=8, lens="1,37,214,64,9,128,65,150", fused=True, hq=32),
        # two 32K prompts of the 8B shape (one ends inside a block)
        dict(name="store_8b_32k_x2", kind="store", hkv=8, lens="32768,32741", fused=False, hq=32),
        # --- fetch ---
        # four sequences of a few thousand tokens leave the cache (another tier takes them)
        dict(name="fetch_mixed", kind="fetch", hkv=8, lens="2067,5003,640,1", hq=32),
        # two 64K sequences
        dict(name="fetch_64k_x2", kind="fetch", hkv=8, lens="65536,65499", hq=64),
        # --- attend ---
        # one sequence of 2K on a small model: the smallest step, where latency counts
        dict(name="attend_2k", kind="attend", hq=8, hkv=8, lens="2067"),
        # an 8B-shaped layer at 32K, one sequence: the ordinary interactive step
        dict(name="attend_8b_32k", kind="attend", hq=32, hkv=8, lens="32768"),
        # the same layer serving eight sequences of different lengths, one of them about to
        # close a block
        dict(name="attend_8b_b8", kind="attend", hq=32, hkv=8,
             lens="32768,30001,16383,24576,32700,8191,20480,29999"),
        # a 70B-shaped layer, a large batch with one long sequence, short ones and empty
        # places (-1)
        dict(name="attend_70b_b32", kind="attend", hq=64, hkv=8,
             lens="131072,0,63,64,1000,-1,20000,32768,5,4095,16000,127,9000,40000,2067,300,"
                  "-1,12345,65535,777,8192,6400,1,30000,25000,11111,2222,33333,4444,5555,-1,18000"),
    ]


_HEADS = [(8, 8), (32, 8), (64, 8), (16, 2), (28, 4)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges of listed(), without a name."""
    kind = rng.choice(["prompt", "prompt", "store", "fetch", "attend", "attend"])
    hq, hkv = rng.choice(_HEADS)
    n = _log_int(rng, 1, 32)
    if kind == "prompt":
        # prompts of 1 to 32K tokens; together not more work than the largest listed case
        lens, room = [], 32768.0 ** 2 * 32
        for _ in range(n):
            t = min(_log_int(rng, 1, 32768), int(math.sqrt(room / hq)))
            if t < 1:
                break
            lens.append(t)
            room -= t * t * hq
        fused = hq > 8 and rng.random() < 0.5
        return dict(kind=kind, hq=hq, hkv=hkv, lens=",".join(map(str, lens)), fused=fused)
    room = (65509 if kind == "store" else 131035) * 8 // hkv
    if kind == "attend":
        room = 470000 * 8 // hkv
    lens = []
    for _ in range(n):
        if kind == "attend" and n > 1 and rng.random() < 0.1:
            lens.append(-1)
            continue
        t = min(_log_int(rng, 1, 131072 if kind == "attend" else 65536), room)
        if t < 1:
            break
        lens.append(t)
        room -= t
    c = dict(kind=kind, hq=hq, hkv=hkv, lens=",".join(map(str, lens)))
    if kind == "store":
        c["fused"] = hq > 8 and rng.random() < 0.5
    return c


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def work(case):
    lens, hq, hkv = _lens(case), case["hq"], case["hkv"]
    if case["kind"] == "prompt":
        return {"bytes": sum(lens) * (2 * hq + 2 * hkv) * D * 2,
                "flops": 4 * D * hq * sum(t * (t + 1) // 2 for t in lens)}
    if case["kind"] in ("store", "fetch"):
        whole = sum(t // BLOCK * BLOCK for t in lens)
        tail = sum(lens) - whole
        cache = hkv * (whole * 2 * D + whole // BLOCK * 8 + tail * 4 * D)
        rows = sum(lens) * hkv * 4 * D
        # store: the rows are read, the cache is written, the values come out
        return {"bytes": rows + cache if case["kind"] == "fetch" else 2 * rows + cache,
                "flops": 2 * sum(lens) * hkv * 2 * D}
    live = [t for t in lens if t >= 0]
    cache = sum(t // BLOCK * (BLOCK * 2 * D + 8) + t % BLOCK * 4 * D for t in live) * hkv
    return {"bytes": cache + len(live) * (2 * hq + 4 * hkv) * D * 2,
            "flops": 4 * D * hq * sum(t + 1 for t in live)}


# ------------------------------------------------------------------ inputs
def _cu(lens):
    cu = [0]
    for t in lens:
        cu.append(cu[-1] + t)
    return cu


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _packed_rows(case, g):
    """q, k, v [tokens, heads, d] bf16: normal keys and values, queries drawn towards one
    direction per KV head that some keys share (heads attend to a few tokens sharply)."""
    hq, hkv, total = case["hq"], case["hkv"], sum(_lens(case))
    if case.get("fused"):
        buf = _normal(g, total, hq + 2 * hkv, D).bfloat16()
        q, k, v = buf[:, :hq], buf[:, hq:hq + hkv], buf[:, hq + hkv:]
    else:
        q, k, v = (_normal(g, total, h, D).bfloat16() for h in (hq, hkv, hkv))
    u = _normal(g, hkv, D)
    u /= u.norm(dim=1, keepdim=True)
    q += (3.0 * u).repeat_interleave(hq // hkv, dim=0).bfloat16()
    mark = (torch.rand(total, hkv, 1, generator=g, device="cuda") < 0.02).float()
    k += (mark * (12.0 * u)).bfloat16()
    return q, k, v


def _cache_tensors(case, g, fill):
    """The tensors of a cache whose sequences have the case's lengths, pages in no order."""
    lens, hkv = _lens(case), case["hkv"]
    n_cols = max(max(lens), 0) // BLOCK + 1
    blocks = [max(t, -1) // BLOCK + 1 for t in lens]     # the open block's page included
    n_pages = sum(blocks) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), n_cols), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, b in enumerate(blocks):
        table[s, :b] = order[at:at + b]
        at += b
    c = dict(table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for name, shape in (("k_codes", (n_pages, hkv, BLOCK, D)), ("v_codes", (n_pages, hkv, D, BLOCK))):
        c[name] = torch.zeros(shape, dtype=torch.int8, device="cuda")
        sc = torch.full((n_pages, hkv), MIN_SCALE, dtype=torch.float32, device="cuda")
        if fill:
            for a in range(0, n_pages, 1024):
                x = _normal(g, *((min(1024, n_pages - a),) + shape[1:]))
                s = x.abs().amax(dim=(2, 3)) / 127.0
                sc[a:a + 1024] = s
                c[name][a:a + 1024] = torch.round(x / s[:, :, None, None]).clamp_(-127, 127).to(torch.int8)
        c[name[0] + "_scale"] = sc
    for name in ("k_tail", "v_tail"):
        x = _normal(g, len(lens), hkv, BLOCK, D)
        c[name] = x.bfloat16()
    return c


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 17)
    lens, hq, hkv = _lens(case), case["hq"], case["hkv"]
    st = dict(case=case, lens=lens)
    if case["kind"] in ("prompt", "store"):
        st["q"], st["k"], st["v"] = _packed_rows(case, g)
    if case["kind"] != "attend":
        st["cu_host"] = _cu(lens)
        st["cu"] = torch.tensor(st["cu_host"], dtype=torch.int32, device="cuda")
    if case["kind"] != "prompt":
        st["cache"] = _cache_tensors(case, g, fill=case["kind"] != "store")
    if case["kind"] == "attend":
        st["q"] = (2.0 * _normal(g, len(lens), hq, D)).bfloat16()
        st["k_new"], st["v_new"] = (_normal(g, len(lens), hkv, D).bfloat16() for _ in range(2))
        st["out"] = torch.zeros(len(lens), hq, D, dtype=torch.bfloat16, device="cuda")
        # the sequences whose open block this token fills, and the page it goes to
        st["filled"] = [s for s, t in enumerate(lens) if t >= 0 and t % BLOCK == BLOCK - 1]
        st["filled_pages"] = torch.stack(
            [st["cache"]["table"][s, lens[s] // BLOCK] for s in st["filled"]]).long() if st["filled"] else None
    elif case["kind"] == "prompt":
        st["out"] = torch.zeros(sum(lens), hq, D, dtype=torch.bfloat16, device="cuda")
    else:
        st["k_out"], st["v_out"] = (torch.zeros(sum(lens), hkv, D, dtype=torch.bfloat16, device="cuda")
                                    for _ in range(2))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own and "cache" in st:
        import paper_2608_05326_amd as qv
        c = st["cache"]
        cfg = qv.BlockConfig(batch=len(st["lens"]), num_q_heads=case["hq"], num_kv_heads=case["hkv"],
                             max_context=c["table"].shape[1] * BLOCK, num_pages=c["k_codes"].shape[0])
        bc = qv.BlockCache(cfg)
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


def _own_prompt(st):
    import paper_2608_05326_amd as qv
    qv.prompt_attend(st["q"], st["k"], st["v"], st["cu"], st["out"])
    return st["out"]


def _own_store(st):
    st["handle"].store(0, st["k"], st["v"], st["cu"])
    return _own_fetch(st)


def _own_fetch(st):
    st["handle"].fetch(0, st["k_out"], st["v_out"], st["cu"])
    return st["k_out"], st["v_out"]


def _own_attend(st):
    st["handle"].attend(0, st["q"], st["k_new"], st["v_new"], st["out"])
    return _attend_outputs(st)


def _attend_outputs(st):
    """The attention output, the open blocks, and the values of the blocks just closed."""
    c = st["cache"]
    res = [st["out"], c["k_tail"], c["v_tail"]]
    p = st["filled_pages"]
    if p is not None:
        res.append(c["k_codes"][p].float() * c["k_scale"][p][:, :, None, None])
        res.append(c["v_codes"][p].float() * c["v_scale"][p][:, :, None, None])
    return tuple(res)


def _softmax_rows(s):
    e = torch.exp(s - s.amax(dim=-1, keepdim=True))
    return e / e.sum(dim=-1, keepdim=True)


def _plain_prompt(st):
    hq, hkv = st["case"]["hq"], st["case"]["hkv"]
    g, rows = hq // hkv, 1024
    for a, b in zip(st["cu_host"], st["cu_host"][1:]):
        q = st["q"][a:b].float().view(b - a, hkv, g, D)
        k = st["k"][a:b].float().permute(1, 2, 0).contiguous()    # [hkv, d, t]
        v = st["v"][a:b].float().transpose(0, 1).contiguous()     # [hkv, t, d]
        pos = torch.arange(b - a, device="cuda")
        for r in range(0, b - a, rows):
            e = min(r + rows, b - a)
            qr = q[r:e].permute(1, 2, 0, 3).reshape(hkv, g * (e - r), D)
            s = (qr @ k[:, :, :e].contiguous()).view(hkv, g, e - r, e) / math.sqrt(D)
            s.masked_fill_(pos[None, :e] > pos[r:e, None], -math.inf)
            o = _softmax_rows(s).view(hkv, g * (e - r), e) @ v[:, :e].contiguous()
            st["out"][a + r:a + e] = o.view(hkv, g, e - r, D).permute(2, 0, 1, 3).reshape(e - r, hq, D)
    return st["out"]


def _quantize(x):
    """Blocks [..., 64, d] -> int8 codes, fp32 scales [...]: half-step decisions in 64 bits."""
    s = (x.float().abs().amax(dim=(-2, -1)).double() / 127.0).float().clamp_min(MIN_SCALE)
    return torch.round(x.double() / s.double()[..., None, None]).to(torch.int8), s


def _close(c, pages, k, v):
    """Blocks k, v [n, H_kv, 64, d] into the pages."""
    c["k_codes"][pages], c["k_scale"][pages] = _quantize(k)
    codes, c["v_scale"][pages] = _quantize(v)
    c["v_codes"][pages] = codes.transpose(-1, -2)


def _plain_store(st):
    c = st["cache"]
    for s, (a, b) in enumerate(zip(st["cu_host"], st["cu_host"][1:])):
        n = (b - a) // BLOCK
        k, v = st["k"][a:b].transpose(0, 1), st["v"][a:b].transpose(0, 1)     # [hkv, t, d]
        if n:
            def blocks(x):
                return x[:, :n * BLOCK].reshape(-1, n, BLOCK, D).transpose(0, 1)
            _close(c, c["table"][s, :n].long(), blocks(k), blocks(v))
        c["k_tail"][s, :, :b - a - n * BLOCK] = k[:, n * BLOCK:]
        c["v_tail"][s, :, :b - a - n * BLOCK] = v[:, n * BLOCK:]
    return _plain_fetch(st)


def _sequence(c, s, t):
    """fp32 keys and values [H_kv, t, d] of sequence s."""
    n = t // BLOCK
    p = c["table"][s, :n].long()
    k = (c["k_codes"][p].float() * c["k_scale"][p][:, :, None, None]).transpose(0, 1)
    v = (c["v_codes"][p].float() * c["v_scale"][p][:, :, None, None]).permute(1, 0, 3, 2)
    hkv = k.shape[0]
    return [torch.cat([x.reshape(hkv, n * BLOCK, D), c[tail][s, :, :t - n * BLOCK].float()], dim=1)
            for x, tail in ((k, "k_tail"), (v, "v_tail"))]


def _plain_fetch(st):
    for s, (a, b) in enumerate(zip(st["cu_host"], st["cu_host"][1:])):
        k, v = _sequence(st["cache"], s, b - a)
        st["k_out"][a:b] = k.transpose(0, 1)
        st["v_out"][a:b] = v.transpose(0, 1)
    return st["k_out"], st["v_out"]


def _plain_attend(st):
    c, hq, hkv = st["cache"], st["case"]["hq"], st["case"]["hkv"]
    for s, t in enumerate(st["lens"]):
        if t < 0:
            continue
        c["k_tail"][s, :, t % BLOCK] = st["k_new"][s]
        c["v_tail"][s, :, t % BLOCK] = st["v_new"][s]
        n = t // BLOCK * BLOCK
        k, v = _sequence(c, s, n)
        k = torch.cat([k, c["k_tail"][s, :, :t - n + 1].float()], dim=1)
        v = torch.cat([v, c["v_tail"][s, :, :t - n + 1].float()], dim=1)
        q = st["q"][s].float().view(hkv, hq // hkv, D)
        p = _softmax_rows(q @ k.transpose(1, 2).contiguous() / math.sqrt(D))
        st["out"][s] = (p @ v).view(hq, D)
    if st["filled"]:
        _close(c, st["filled_pages"], c["k_tail"][st["filled"]], c["v_tail"][st["filled"]])
    return _attend_outputs(st)


_PLAIN = dict(prompt=_plain_prompt, store=_plain_store, fetch=_plain_fetch, attend=_plain_attend)
_OWN = dict(prompt=_own_prompt, store=_own_store, fetch=_own_fetch, attend=_own_attend)


# --------------------------------------------------- results in 64 bits
def _exact_attention(q, k, v, first):
    """q [n, d] at positions first .. first + n - 1, k, v [t, d]: one head in float64."""
    s = q.double() @ k.double().t().contiguous() / D ** 0.5
    pos = torch.arange(first, first + q.shape[0], device="cuda")[:, None]
    s = torch.where(torch.arange(k.shape[0], device="cuda")[None] <= pos, s, -math.inf)
    return torch.softmax(s, dim=1) @ v.double()


def _exact_values(block):
    """[64, d] of one block -> the float64 values its codes stand for."""
    x = block.double()
    scale = max((x.abs().max() / 127.0).float().item(), MIN_SCALE)
    return torch.round(x / scale) * scale


def _exact_rows(rows):
    """[t, d] of one sequence and head -> the values a cache holds for them."""
    x = rows.double()
    n = x.shape[0] // BLOCK
    b = x[:n * BLOCK].reshape(n, BLOCK * D)
    scale = (b.abs().amax(dim=1, keepdim=True) / 127.0).float().clamp_min(MIN_SCALE).double()
    return torch.cat([(torch.round(b / scale) * scale).view(-1, D), x[n * BLOCK:]])


def exact(case, seed):
    """What run returns for these inputs, in float64 from the definitions."""
    st = _inputs(case, seed)
    hq, hkv, lens = case["hq"], case["hkv"], st["lens"]
    group = hq // hkv
    if case["kind"] == "prompt":
        out = torch.zeros(sum(lens), hq, D, dtype=torch.float64, device="cuda")
        for start, t in zip(st["cu_host"], lens):
            for h in range(hq):
                k, v = (st[x][start:start + t, h // group] for x in "kv")
                for r in range(0, t, 4096):
                    e = min(r + 4096, t)
                    out[start + r:start + e, h] = _exact_attention(st["q"][start + r:start + e, h], k[:e], v[:e], r)
        return out
    if case["kind"] == "store":
        res = []
        for x in (st["k"], st["v"]):
            o = torch.zeros(sum(lens), hkv, D, dtype=torch.float64, device="cuda")
            for start, t in zip(st["cu_host"], lens):
                for h in range(hkv):
                    o[start:start + t, h] = _exact_rows(x[start:start + t, h])
            res.append(o)
        return tuple(res)
    c = st["cache"]

    def held(name, s, h, t):
        """Tokens 0 .. t - 1 of sequence s and KV head h, [t, d]."""
        n = t // BLOCK
        pages = c["table"][s, :n].long()
        codes = c[name + "_codes"][pages, h].double()
        if name == "v":
            codes = codes.transpose(1, 2)
        whole = (codes * c[name + "_scale"][pages, h].double().view(n, 1, 1)).reshape(n * BLOCK, D)
        return torch.cat([whole, c[name + "_tail"][s, h, :t - n * BLOCK].double()])

    if case["kind"] == "fetch":
        res = []
        for name in "kv":
            o = torch.zeros(sum(lens), hkv, D, dtype=torch.float64, device="cuda")
            for s, (start, t) in enumerate(zip(st["cu_host"], lens)):
                for h in range(hkv):
                    o[start:start + t, h] = held(name, s, h, t)
            res.append(o)
        return tuple(res)
    out = torch.zeros(len(lens), hq, D, dtype=torch.float64, device="cuda")
    tails = [c[x].double().clone() for x in ("k_tail", "v_tail")]
    for s, t in enumerate(lens):
        if t < 0:
            continue
        for h in range(hkv):
            kv = [torch.cat([held(name, s, h, t), st[name + "_new"][s, h].double()[None]]) for name in "kv"]
            heads = slice(h * group, (h + 1) * group)
            logits = st["q"][s, heads].double() @ kv[0].t().contiguous() / D ** 0.5
            out[s, heads] = torch.softmax(logits, dim=1) @ kv[1]
            for tail, name in zip(tails, "kv"):
                tail[s, h, t % BLOCK] = st[name + "_new"][s, h].double()
    res = [out] + tails
    if st["filled"]:
        for tail, turn in zip(tails, (False, True)):
            vals = torch.stack([torch.stack([_exact_values(tail[s, h]) for h in range(hkv)])
                                for s in st["filled"]])
            res.append(vals.transpose(-1, -2) if turn else vals)
    return tuple(res)
