"""Cases of the cache operators: an 8-bit cache (quantise, append, attend) and eviction by accumulated attention weight.

A cache of one layer is a pool of rows [total_rows, 128]; segment s = (sequence, KV head) owns rows
[off[s], off[s] + cap[s]) of which the first len[s] are valid; offsets and capacities are multiples of 128.
The 8-bit cache holds complete blocks of 64 rows as 8-bit codes with one fp32 scale per block (K and V apart) and the
rows of the last, unfinished block as bf16 in a tail of 64 rows per segment.
"""
import math

import torch

own = False

D, BLOCK, ALIGN = 128, 64, 128
TOP = {"e4m3": 448.0, "int8": 127.0}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one layer, 4096 tokens, half of the heads cut to 256: the smallest step, where latency counts
        {"name": "q8 attention 4k", "op": "q8_attn", "B": 1, "Hq": 32, "Hkv": 8, "n": 4096, "budget": 256, "share": 0.5,
         "type": "e4m3", "out": "fp32"},
        # one sequence of 128K tokens, adaptive heads at 90 %, consistent heads at 2048: a long prompt being answered
        {"name": "q8 attention 128k", "op": "q8_attn", "B": 1, "Hq": 32, "Hkv": 8, "n": 117964, "budget": 2048, "share": 0.6,
         "type": "int8", "out": "bf16"},
        # batched serving, 16 sequences of 64K tokens with ragged lists: the largest
        {"name": "q8 attention 16x64k", "op": "q8_attn", "B": 16, "Hq": 32, "Hkv": 8, "n": 65536, "budget": 1024, "share": 0.55,
         "type": "e4m3", "out": "bf16"},
        # a group of seven query heads over 256K tokens, an odd length
        {"name": "q8 attention gqa7 256k", "op": "q8_attn", "B": 1, "Hq": 28, "Hkv": 4, "n": 262143, "budget": 4096, "share": 0.5,
         "type": "e4m3", "out": "fp32"},
        # a decode step: the new token's row is appended (one list in eight completes a block by it), then attended to
        {"name": "q8 step 32k", "op": "q8_step", "B": 1, "Hq": 32, "Hkv": 8, "n": 32768, "budget": 1024, "share": 0.5,
         "type": "e4m3", "out": "bf16"},
        # the same for many short lists of odd lengths
        {"name": "q8 step 16x1k", "op": "q8_step", "B": 16, "Hq": 32, "Hkv": 8, "n": 1021, "budget": 300, "share": 0.4,
         "type": "int8", "out": "fp32"},
        # the end of a short prompt: its cache goes to 8 bits
        {"name": "q8 quantize 4k", "op": "q8_quantize", "B": 1, "Hkv": 8, "n": 4099, "budget": 256, "share": 0.5, "type": "int8"},
        # the end of a 128K prompt
        {"name": "q8 quantize 128k", "op": "q8_quantize", "B": 1, "Hkv": 8, "n": 117964, "budget": 2048, "share": 0.4,
         "type": "e4m3"},
        # decode steps that keep count of what every cached row is worth: one sequence, and a batch
        {"name": "weighted attention 32k", "op": "weighted", "B": 1, "Hq": 32, "Hkv": 8, "n": 32768, "budget": 1024, "share": 0.5,
         "decay": 1.0, "out": "fp32"},
        {"name": "weighted attention 8x64k", "op": "weighted", "B": 8, "Hq": 28, "Hkv": 4, "n": 65521, "budget": 1024, "share": 0.5,
         "decay": 0.97, "out": "bf16"},
        # consistent heads that have grown by 256 tokens go back to their budget
        {"name": "evict 1280 to 1024", "op": "evict", "B": 1, "Hkv": 8, "n": 1280, "keep": 1024, "sink": 4, "local": 64, "share": 0.5},
        # a batch of long adaptive heads is cut to half
        {"name": "evict 8x48k", "op": "evict", "B": 8, "Hkv": 8, "n": 49100, "keep": 24576, "sink": 4, "local": 256, "share": 0.6},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["q8_attn", "q8_attn", "q8_step", "q8_quantize", "weighted", "evict"])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    B = _log(rng, 1, 16)
    G = rng.randint(1, 8)
    n = _log(rng, 1, min(262144, (4 if op in ("q8_attn", "q8_step", "q8_quantize") else 2) * 2 ** 20 // (B * Hkv)))
    c = {"op": op, "B": B, "Hkv": Hkv, "n": n, "share": round(rng.uniform(0.0, 0.9), 2)}
    if op == "evict":
        c.update(keep=rng.randint(0, n), sink=rng.randint(0, 8), local=rng.randint(0, 300))
        return c
    c["budget"] = _log(rng, 1, 4096)
    if op != "q8_quantize":
        c.update(Hq=Hkv * G, out=rng.choice(["bf16", "fp32"]))
    if op == "weighted":
        c["decay"] = rng.choice([1.0, 0.9, 0.5])
    else:
        c["type"] = rng.choice(["e4m3", "int8"])
    return c


# ---------------------------------------------------------------------------------------------- shapes
def _lens(c):
    """Rows of every segment: a `share` of the heads is short (`budget` rows, or none to cut for an eviction); lengths differ from
    sequence to sequence as lists that have been appended to for different times do."""
    lens, k = [], c["Hkv"]
    short = round(c["share"] * k)
    for b in range(c["B"]):
        n = max(1, c["n"] - (b * 37) % max(1, min(c["n"], 611)))
        for h in range(k):
            is_short = (h * 5 + b * 3) % k < short
            if c["op"] == "evict":
                lens.append(max(1, n // 7) if is_short else n)
            elif c["op"] == "q8_step" and h == 0:
                lens.append(n // BLOCK * BLOCK + BLOCK - 1)  # this list's block is completed by the step
            else:
                lens.append(min(n, c["budget"]) if is_short else n)
    return lens


def _mask(c):
    """Eviction looks at every head but the short ones."""
    k, short = c["Hkv"], round(c["share"] * c["Hkv"])
    return [0 if (h * 5 + b * 3) % k < short else 1 for b in range(c["B"]) for h in range(k)]


def _kept(c):
    kept = []
    for n, m in zip(_lens(c), _mask(c)):
        forced = c["sink"] + c["local"]
        kept.append(n if not m or c["keep"] >= n or forced >= n else max(c["keep"], forced))
    return kept


def _layout(lens, room):
    off, cap, at = [], [], 0
    for n in lens:
        r = (n + room + ALIGN - 1) // ALIGN * ALIGN
        off.append(at)
        cap.append(r)
        at += r
    return off, cap, at


def work(case):
    c, lens = case, _lens(case)
    rows = sum(lens)
    full = sum(n // BLOCK * BLOCK for n in lens)
    scales = full // BLOCK * 8
    if c["op"] == "q8_quantize":
        return {"bytes": 512 * rows + 256 * full + 512 * (rows - full) + scales, "flops": 2 * 2 * D * full}
    if c["op"] == "evict":
        kept = sum(_kept(c))
        scored = sum(n for n, k in zip(lens, _kept(c)) if k < n)
        return {"bytes": 1024 * kept + 4 * scored + 8 * kept, "flops": 0}
    io = c["B"] * c["Hq"] * D * (2 + (2 if c["out"] == "bf16" else 4)) + 4 * c["B"] * c["Hq"]
    g = c["Hq"] // c["Hkv"]
    if c["op"] == "weighted":
        return {"bytes": 512 * rows + 8 * rows + io, "flops": 4 * g * D * rows}
    if c["op"] == "q8_step":
        # the lists after the append; a block that the step completes is read as bf16, and its codes are written
        new = [n + 1 for n in lens]
        done = sum(n % BLOCK == 0 for n in new)
        seen = sum(n // BLOCK * BLOCK for n in new)
        held = seen - done * BLOCK
        tail = sum(new) - held
        return {"bytes": 256 * held + held // BLOCK * 8 + 512 * tail + 512 * len(new) + done * BLOCK * 256 + io, "flops": 4 * g * D * sum(new)}
    return {"bytes": 256 * full + scales + 512 * (rows - full) + io, "flops": 4 * g * D * rows}


# ---------------------------------------------------------------------------------------------- inputs
def _encode(x, kind):
    """Blocks [n, 64, 128] -> (codes, scale [n]).  x * M and the largest magnitude are bf16 numbers times an integer: the quotient of the two is
    never nearer to the border of two codes than 2^-17 of itself unless it lies on it, so that 32 bits round it as the reals do."""
    x = x.float()
    a = x.abs().amax(dim=(1, 2))
    scale = a / TOP[kind]
    r = x * TOP[kind] / torch.where(a > 0, a, torch.ones_like(a))[:, None, None]
    codes = r.to(torch.float8_e4m3fn) if kind == "e4m3" else torch.round(r).to(torch.int8)
    return codes, scale


def _rows(total, gen, dev):
    return torch.randn(total, D, generator=gen, device=dev, dtype=torch.bfloat16)


def _padded(off, lens, dev):
    """[S, longest] pool rows of every segment, and which of them are there."""
    at = torch.arange(max(max(lens), 1), device=dev)
    ok = at[None] < torch.tensor(lens, device=dev)[:, None]
    return torch.where(ok, torch.tensor(off, device=dev)[:, None] + at[None], 0), ok


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    lens = _lens(c)
    S = len(lens)
    off, cap, total = _layout(lens, 64)
    st = {"c": c, "lens": lens, "off": off, "cap": cap, "total": total}
    q8 = c["op"] in ("q8_attn", "q8_step")
    kind = c.get("type")
    code_type = torch.float8_e4m3fn if kind == "e4m3" else torch.int8
    if own:
        import numpy as np
        import paper_2608_30295_b200 as ck
        st["ck"] = ck
    idx, ok = _padded(off, lens, dev)
    st["idx"], st["ok"] = idx, ok
    st["pool_seg"] = torch.repeat_interleave(torch.arange(S, device=dev), torch.tensor(cap, device=dev))
    st["pool_row"] = torch.arange(total, device=dev) - torch.tensor(off, device=dev)[st["pool_seg"]]
    seg_len = torch.tensor(lens, dtype=torch.int32, device=dev)
    valid = st["pool_row"] < seg_len[st["pool_seg"]]

    # queries and keys share a direction in every segment: a few rows take much of the attention, as they do in a model
    heavy = torch.randn(S, D, generator=gen, device=dev)
    heavy = heavy / heavy.norm(dim=1, keepdim=True) * (2 * D ** 0.25)
    k, v = _rows(total, gen, dev), _rows(total, gen, dev)
    hit = (torch.rand(S, 16, generator=gen, device=dev) * torch.tensor(lens, device=dev)[:, None]).long()
    at = (hit + torch.tensor(off, device=dev)[:, None]).reshape(-1)
    k[at] = (k[at].float() + heavy.repeat_interleave(16, 0)).to(torch.bfloat16)
    if "Hq" in c:
        q = torch.randn(c["B"], c["Hq"], D, generator=gen, device=dev)
        st["q"] = (q + heavy.reshape(c["B"], c["Hkv"], 1, D).expand(-1, -1, c["Hq"] // c["Hkv"], -1).reshape(q.shape)).to(torch.bfloat16)
        st["out"] = torch.empty(c["B"], c["Hq"], D, device=dev, dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32)
        st["lse"] = torch.empty(c["B"], c["Hq"], device=dev)

    if not q8:
        # what lies behind a list is no part of it
        k[~valid], v[~valid] = float("nan"), float("nan")
        if own:
            src = ck.Cache(c["B"], c["Hkv"], lens, 64, dev)
            src.k_pool.copy_(k)
            src.v_pool.copy_(v)
            src.set_lengths(lens)
            st["src"] = src
        else:
            st["k"], st["v"] = k, v
    if c["op"] == "weighted" or c["op"] == "evict":
        w = torch.rand(total, generator=gen, device=dev).pow(4) * valid
        if c["op"] == "evict":
            w = torch.where(torch.rand(total, generator=gen, device=dev) < 0.1, w.mul(64).floor() / 64, w)  # rows that tie
        st["w"] = w
    if c["op"] == "weighted" and own:
        st["plan"] = ck.DecodePlan(src, ck.catekv_decode_num_ctas())
        ck.catekv_decode_plan(src, st["plan"])
        st["ws"] = ck.decode_weighted_workspace(src, c["Hq"], st["plan"])
    if c["op"] == "evict":
        kept = _kept(c)
        doff, dcap, dtotal = _layout(kept, 64)
        st.update(kept=kept, doff=doff, dtotal=dtotal, dw=torch.full((dtotal,), 7.0, device=dev))
        st["kidx"] = torch.full((S, max(kept)), -1, dtype=torch.int32, device=dev)
        if own:
            dst = ck.Cache(c["B"], c["Hkv"], kept, 64, dev)
            dst.k_pool.zero_()
            dst.v_pool.zero_()
            st["dst"], st["mask"] = dst, np.array(_mask(c), dtype=np.uint8)
            st["ws"] = ck.evict_workspace(src)
        else:
            st["dk"] = torch.zeros(dtotal, D, dtype=torch.bfloat16, device=dev)
            st["dv"], st["dlen"] = torch.zeros_like(st["dk"]), torch.zeros(S, dtype=torch.int32, device=dev)
            st["mask"] = torch.tensor(_mask(c), device=dev, dtype=torch.bool)
            st["n"], st["t"] = torch.tensor(lens, device=dev), torch.tensor(kept, device=dev)
            there = torch.arange(max(kept), device=dev)[None] < st["t"][:, None]
            st["there"] = there
            st["to"] = (torch.tensor(doff, device=dev)[:, None] + torch.arange(max(kept), device=dev)[None])[there]
    if q8 or c["op"] == "q8_quantize":
        if own:
            cache = ck.Q8Cache(c["B"], c["Hkv"], lens, 64, ck.Q8_E4M3 if kind == "e4m3" else ck.Q8_INT8, dev)
            t = {x: getattr(cache, x) for x in ("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail", "seg_len_dev")}
            st["cache"] = cache
        else:
            t = {x: torch.empty(total, D, dtype=torch.int8, device=dev).view(code_type) for x in ("k_pool", "v_pool")}
            t.update({x: torch.empty(total // BLOCK, device=dev) for x in ("k_scale", "v_scale")})
            t.update({x: torch.empty(S, BLOCK, D, dtype=torch.bfloat16, device=dev) for x in ("k_tail", "v_tail")})
            t["seg_len_dev"] = torch.empty(S, dtype=torch.int32, device=dev)
        for x in t.values():
            x.view(torch.int8).zero_()
        st["t"] = {**st["t"], **t} if isinstance(st.get("t"), dict) else t
    if q8:
        t, full = st["t"], [n // BLOCK * BLOCK for n in lens]
        block = torch.arange(total // BLOCK, device=dev) * BLOCK
        there = st["pool_row"][block] < torch.tensor(full, device=dev)[st["pool_seg"][block]]
        left = torch.tensor([n % BLOCK for n in lens], device=dev)[:, None] > torch.arange(BLOCK, device=dev)[None]
        last = torch.tensor([o + f for o, f in zip(off, full)], device=dev)[:, None] + torch.arange(BLOCK, device=dev)[None]
        for x, name in ((k, "k"), (v, "v")):
            codes, scale = _encode(x.reshape(-1, BLOCK, D), kind)
            codes = codes.view(torch.int8)
            codes[~there] = 127  # behind the lists: NaN as e4m3
            t[name + "_pool"].view(torch.int8).copy_(codes.reshape(total, D))
            t[name + "_scale"].copy_(torch.where(there, scale, float("nan")))
            t[name + "_tail"].copy_(torch.where(left[..., None], x[last.clamp(max=total - 1)], float("nan")))
        t["seg_len_dev"].copy_(seg_len)
        st["len0"] = seg_len
        if c["op"] == "q8_step":
            st["idx"], st["ok"] = _padded(off, [n + 1 for n in lens], dev)
            st["kn"], st["vn"] = (torch.randn(c["B"], c["Hkv"], D, generator=gen, device=dev, dtype=torch.bfloat16) for _ in range(2))
        if own:
            cache.set_lengths(lens)
            st["len0_host"] = cache.seg_len.copy()
            st["plan"] = ck.DecodePlan(cache, ck.catekv_q8_decode_num_ctas())
            ck.catekv_q8_decode_plan(cache, st["plan"])
    return st


# ---------------------------------------------------------------------------------------------- one pass
def _codes(t, kind):
    """A pool's bytes as the numbers they are."""
    return t.view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8)


def _attend(q, k, v, ok):
    """q [S, G, D], k and v [S, L, D] fp32, ok [S, L] -> out [S, G, D], lse [S, G], p [S, G, L]."""
    x = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(D)
    x = x.masked_fill(~ok[:, None], float("-inf"))
    m = x.amax(dim=2, keepdim=True)
    e = torch.exp(x - torch.where(m > float("-inf"), m, 0.0))
    s = e.sum(dim=2, keepdim=True)
    p = e / torch.where(s > 0, s, 1.0)
    return torch.matmul(p, v), (m + torch.log(s)).squeeze(2), p


def _plain_q8_cache(t, kind, lens_dev, idx):
    """K and V of the whole lists as fp32 [S, L + 64, D] (the blocks, then the tail) and which rows are there."""
    n = lens_dev[:, None].long()
    ok = torch.cat([torch.arange(idx.shape[1], device=idx.device)[None] < n // BLOCK * BLOCK,
                    torch.arange(BLOCK, device=idx.device)[None] < n % BLOCK], 1)
    kv = []
    for x in ("k", "v"):
        y = _codes(t[x + "_pool"], kind).view(torch.int8)[idx].view(_codes(t[x + "_pool"], kind).dtype).float() * t[x + "_scale"][idx // BLOCK][..., None]
        y = torch.cat([y, t[x + "_tail"].float()], 1)
        kv.append(y.masked_fill_(~ok[..., None], 0.0))
    return kv[0], kv[1], ok


def run(state):
    st, c = state, state["c"]
    if c["op"] == "q8_quantize":
        return _run_quantize(st, c)
    if c["op"] == "evict":
        return _run_evict(st, c)
    if c["op"] == "weighted":
        return _run_weighted(st, c)
    return _run_q8_attention(st, c)


def _run_quantize(st, c):
    t = st["t"]
    if own:
        st["ck"].catekv_q8_quantize(st["src"], st["cache"])
    else:
        lens = torch.tensor(st["lens"], device="cuda")
        block = torch.arange(st["total"] // BLOCK, device="cuda") * BLOCK
        there = st["pool_row"][block] < (lens // BLOCK * BLOCK)[st["pool_seg"][block]]
        left = torch.arange(BLOCK, device="cuda")[None] < (lens % BLOCK)[:, None]
        last = torch.tensor(st["off"], device="cuda")[:, None] + (lens // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device="cuda")[None]
        for x in ("k", "v"):
            codes, scale = _encode(torch.where(there[:, None, None], st[x].reshape(-1, BLOCK, D), 0.0), c["type"])
            t[x + "_pool"].view(torch.int8).copy_(torch.where(there[:, None, None], codes.view(torch.int8), t[x + "_pool"].view(torch.int8).reshape(-1, BLOCK, D)).reshape(-1, D))
            t[x + "_scale"].copy_(torch.where(there, scale, t[x + "_scale"]))
            t[x + "_tail"].copy_(torch.where(left[..., None], st[x][last.clamp(max=st["total"] - 1)], t[x + "_tail"]))
        t["seg_len_dev"].copy_(lens)
    return [_codes(t["k_pool"], c["type"]), _codes(t["v_pool"], c["type"]), t["k_scale"], t["v_scale"], t["k_tail"], t["v_tail"], t["seg_len_dev"]]


def _run_q8_attention(st, c):
    t = st["t"]
    step = c["op"] == "q8_step"
    if step:
        t["seg_len_dev"].copy_(st["len0"])  # back to where the step begins, so that it can be run again
    if own:
        ck, cache = st["ck"], st["cache"]
        if step:
            cache.seg_len[:] = st["len0_host"]
            ck.catekv_q8_append(cache, st["kn"], st["vn"])
        ck.catekv_q8_decode_attn(cache, st["q"], st["plan"], st["out"], st["lse"])
    else:
        if step:
            _plain_append(st, c, t)
        k, v, ok = _plain_q8_cache(t, c["type"], t["seg_len_dev"], st["idx"])
        G = c["Hq"] // c["Hkv"]
        o, lse, _ = _attend(st["q"].float().reshape(-1, G, D), k, v, ok)
        st["out"].copy_(o.reshape(st["out"].shape))
        st["lse"].copy_(lse.reshape(st["lse"].shape))
    if step:
        return [st["out"], st["lse"], t["seg_len_dev"], _codes(t["k_pool"], c["type"]), _codes(t["v_pool"], c["type"]), t["k_tail"], t["v_tail"]]
    return [st["out"], st["lse"]]


def _plain_append(st, c, t):
    n = t["seg_len_dev"].long()
    S = n.numel()
    seg = torch.arange(S, device="cuda")
    for x, new in (("k", st["kn"]), ("v", st["vn"])):
        t[x + "_tail"][seg, n % BLOCK] = new.reshape(S, D)
        done = (n % BLOCK == BLOCK - 1)
        codes, scale = _encode(torch.where(done[:, None, None], t[x + "_tail"], 0.0), c["type"])
        block = (torch.tensor(st["off"], device="cuda") + n) // BLOCK
        pool = t[x + "_pool"].view(torch.int8).reshape(-1, BLOCK, D)
        pool[block] = torch.where(done[:, None, None], codes.view(torch.int8), pool[block])
        t[x + "_scale"][block] = torch.where(done, scale, t[x + "_scale"][block])
    t["seg_len_dev"].add_(1)


def _run_weighted(st, c):
    if own:
        st["ck"].catekv_decode_attn_weighted(st["src"], st["q"], st["plan"], st["out"], st["w"], c["decay"], st["ws"], st["lse"])
    else:
        G, ok, idx = c["Hq"] // c["Hkv"], st["ok"], st["idx"]
        k = st["k"][idx].float().masked_fill_(~ok[..., None], 0.0)
        v = st["v"][idx].float().masked_fill_(~ok[..., None], 0.0)
        o, lse, p = _attend(st["q"].float().reshape(-1, G, D), k, v, ok)
        st["out"].copy_(o.reshape(st["out"].shape))
        st["lse"].copy_(lse.reshape(st["lse"].shape))
        row = torch.where(st["pool_row"] < ok.shape[1], st["pool_row"], 0)
        there = ok[st["pool_seg"], row] & (st["pool_row"] < ok.shape[1])
        st["w"].copy_(torch.where(there, c["decay"] * st["w"] + p.mean(dim=1)[st["pool_seg"], row], st["w"]))
    return [st["out"], st["lse"], st["w"]]


def _run_evict(st, c):
    if own:
        ck, dst = st["ck"], st["dst"]
        ck.catekv_evict(st["src"], st["w"], st["mask"], c["keep"], c["sink"], c["local"], dst, st["dw"], st["kidx"], st["ws"])
        return [dst.k_pool, dst.v_pool, st["dw"], dst.seg_len_dev, st["kidx"]]
    n, t, ok, there = st["n"][:, None], st["t"][:, None], st["ok"], st["there"]
    at = torch.arange(ok.shape[1], device="cuda")[None]
    w = torch.where(ok, st["w"][st["idx"]], float("-inf"))
    w = torch.where(ok & ((at < c["sink"]) | (at >= n - c["local"])), float("inf"), w)
    order = torch.sort(w, dim=1, descending=True, stable=True).indices  # ties: lowest index first
    rank = torch.empty_like(order).scatter_(1, order, at.expand_as(order))
    kept = torch.sort(torch.where(rank < t, at, ok.shape[1]), dim=1).values[:, : there.shape[1]]
    st["kidx"].copy_(torch.where(there, kept.int(), st["kidx"]))
    rows = torch.gather(st["idx"], 1, kept.clamp(max=ok.shape[1] - 1))[there]
    st["dk"][st["to"]] = st["k"][rows]
    st["dv"][st["to"]] = st["v"][rows]
    st["dw"].zero_()
    st["dw"][st["to"]] = st["w"][rows]
    st["dlen"].copy_(st["t"])
    return [st["dk"], st["dv"], st["dw"], st["dlen"], st["kidx"]]


# ---------------------------------------------------------------------------------------------- in 64 bits
def _grid64(x, a, kind):
    """round(x M / a) to the type's numbers, ties to even, from the definition of the type."""
    r = x * TOP[kind] / torch.where(a > 0, a, 1.0)
    if kind == "int8":
        return torch.round(r)
    step = torch.exp2(torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3)  # 3 bits behind the leading one; 2^-9 below 2^-6
    return torch.round(r / step) * step


def _blocks64(x, kind):
    x = x.double()
    a = x.abs().amax(dim=(-2, -1), keepdim=True)
    return _grid64(x, a, kind), a / TOP[kind]


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    lens, off = st["lens"], st["off"]
    G = c.get("Hq", c["Hkv"]) // c["Hkv"]
    kind = c.get("type")
    dev = "cuda"
    if c["op"] == "evict":
        rows, to = [], []
        for s, (n, o, t) in enumerate(zip(lens, off, _kept(c))):
            at = torch.arange(n, device=dev)
            if t < n:
                lo, hi = c["sink"], n - c["local"]
                best = torch.sort(st["w"][o + lo:o + hi].double(), descending=True, stable=True).indices[: t - lo - c["local"]] + lo
                at = torch.cat([at[:lo], torch.sort(best).values, at[hi:]])
            rows.append(at + o)
            to.append(torch.arange(t, device=dev) + st["doff"][s])
        rows, to = torch.cat(rows), torch.cat(to)
        k, v = (torch.zeros(st["dtotal"], D, dtype=torch.float64, device=dev) for _ in range(2))
        w = torch.zeros(st["dtotal"], dtype=torch.float64, device=dev)
        k[to], v[to], w[to] = st["k"][rows].double(), st["v"][rows].double(), st["w"][rows].double()
        return [k, v, w, None, None]
    if c["op"] == "q8_quantize":
        outs = []
        for x in ("k", "v"):
            pool = torch.zeros(st["total"], D, dtype=torch.float32, device=dev)  # a code is exact in 32 bits
            scale = torch.zeros(st["total"] // BLOCK, dtype=torch.float64, device=dev)
            tail = torch.zeros(len(lens), BLOCK, D, dtype=torch.float64, device=dev)
            for s, (n, o) in enumerate(zip(lens, off)):
                f = n // BLOCK * BLOCK
                if f:
                    q, sc = _blocks64(st[x][o:o + f].reshape(-1, BLOCK, D), kind)
                    pool[o:o + f] = q.reshape(f, D).float()
                    scale[o // BLOCK:(o + f) // BLOCK] = sc.reshape(-1)
                tail[s, : n - f] = st[x][o + f:o + n].double()
            outs.append((pool.double() if kind == "e4m3" else None, scale, tail))
        return [outs[0][0], outs[1][0], outs[0][1], outs[1][1], outs[0][2], outs[1][2], None]
    q = st["q"].double().reshape(len(lens), G, D)
    out = torch.zeros(len(lens), G, D, dtype=torch.float64, device=dev)
    lse = torch.full((len(lens), G), float("-inf"), dtype=torch.float64, device=dev)
    w = st["w"].double() if c["op"] == "weighted" else None
    for s, (n, o) in enumerate(zip(lens, off)):
        if c["op"] == "weighted":
            k, v = st["k"][o:o + n].double(), st["v"][o:o + n].double()
        else:
            t = st["t"]
            f = n // BLOCK * BLOCK
            parts = []
            for x in ("k", "v"):
                y = _codes(t[x + "_pool"], kind)[o:o + f].float().double().reshape(-1, BLOCK, D) * t[x + "_scale"][o // BLOCK:(o + f) // BLOCK].double()[:, None, None]
                z = t[x + "_tail"][s, : n - f].double()
                if c["op"] == "q8_step":
                    z = torch.cat([z, st["kn" if x == "k" else "vn"].double().reshape(len(lens), D)[s][None]])
                    if z.shape[0] == BLOCK:
                        g, sc = _blocks64(z[None], kind)
                        z = (g * sc)[0]
                parts.append(torch.cat([y.reshape(-1, D), z]))
            k, v = parts
        x = q[s] @ k.T / math.sqrt(D)
        lse[s] = torch.logsumexp(x, dim=1)
        p = torch.exp(x - lse[s][:, None])
        out[s] = p @ v
        if w is not None:
            w[o:o + n] = c["decay"] * w[o:o + n] + p.mean(dim=0)
    out, lse = out.reshape(c["B"], c["Hq"], D), lse.reshape(c["B"], c["Hq"])
    if w is not None:
        return [out, lse, w]
    if c["op"] == "q8_step":
        return [out, lse, None, None, None, None, None]
    return [out, lse]
