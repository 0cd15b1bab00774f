"""Cases of the paged cache's operators: chunks of new tokens (append, attention, taking back) and its pages (fork, compact).

A cache of one layer is a pool of rows [total_rows, 128]; segment s = (sequence, KV head) owns rows
[off[s], off[s] + cap[s]) of which the first len[s] are valid; offsets and capacities are multiples of 128.  Rows from cap[s]
on live in overflow pages of 64 rows: row cap[s] + 64 p + i of segment s is row 64 table[s, p] + i of the overflow pools.
A chunk has n_new[b] tokens of sequence b, on a token axis [n_tokens, heads, 128]: packed one sequence behind the other, or padded.
"""
import math

import torch

own = False

D, PAGE, ALIGN = 128, 64, 128


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of one sequence over a short hybrid cache, as in a decode step: the smallest, where latency counts
        {"name": "attention 1 token 4k", "op": "attn", "B": 1, "Hq": 32, "Hkv": 8, "n": 4096, "budget": 256, "share": 0.5, "T": 1,
         "ragged": 0.0, "grown": 0, "layout": "packed", "out": "fp32"},
        # drafted tokens of sixteen sequences are verified over 64K tokens each: a stream of the whole cache
        {"name": "attention 4 tokens 16x64k", "op": "attn", "B": 16, "Hq": 32, "Hkv": 8, "n": 65536, "budget": 1024, "share": 0.55, "T": 4,
         "ragged": 0.5, "grown": 200, "layout": "padded", "out": "bf16"},
        # a further turn of a conversation, 512 tokens over a 128K prompt and what was generated after it: the largest
        {"name": "attention 512 tokens 128k", "op": "attn", "B": 1, "Hq": 32, "Hkv": 8, "n": 116000, "budget": 2048, "share": 0.6, "T": 512,
         "ragged": 0.0, "grown": 1500, "layout": "packed", "out": "bf16"},
        # a prompt into empty lists
        {"name": "attention 4096 tokens alone", "op": "attn", "B": 1, "Hq": 32, "Hkv": 8, "n": 0, "budget": 0, "share": 0.0, "T": 4096,
         "ragged": 0.0, "grown": 0, "layout": "packed", "out": "bf16"},
        # groups of seven query heads, odd lengths, results in 32 bits
        {"name": "attention 333 tokens gqa7 64k", "op": "attn", "B": 1, "Hq": 28, "Hkv": 4, "n": 65521, "budget": 4096, "share": 0.5, "T": 333,
         "ragged": 0.0, "grown": 77, "layout": "packed", "out": "fp32"},
        # a mixed batch: pieces of prompts beside sequences that decode
        {"name": "attention mixed 8x16k", "op": "attn", "B": 8, "Hq": 32, "Hkv": 8, "n": 16001, "budget": 1024, "share": 0.5, "T": 256,
         "ragged": 1.0, "grown": 130, "layout": "packed", "out": "bf16"},
        # five drafted tokens of sixteen sequences enter the lists and none is accepted
        {"name": "draft 5 tokens 16x4k", "op": "draft", "B": 16, "Hkv": 8, "n": 4000, "budget": 500, "share": 0.4, "T": 5, "ragged": 0.5,
         "grown": 100, "layout": "padded"},
        # pieces of four prompts enter, and the request is given up
        {"name": "draft 4096 tokens 4x32k", "op": "draft", "B": 4, "Hkv": 8, "n": 32700, "budget": 1024, "share": 0.5, "T": 4096,
         "ragged": 0.25, "grown": 300, "layout": "packed"},
        # eight answers to one 32K prompt
        {"name": "fork 8 answers 32k", "op": "fork", "B": 8, "Hkv": 8, "n": 32741, "budget": 1024, "share": 0.5, "keep": 1, "grown": 0},
        # a beam search that has generated for a while: a third of the beams goes on
        {"name": "fork 48 beams", "op": "fork", "B": 48, "Hkv": 8, "n": 2000, "budget": 700, "share": 0.5, "keep": 16, "grown": 421},
        # sequences that have ended leave holes: a few pages, and most of a large pool
        {"name": "compact 8 lists", "op": "compact", "B": 2, "Hkv": 4, "n": 1000, "budget": 1000, "share": 0.0, "grown": 500, "gone": 0.5},
        {"name": "compact 64x8 lists", "op": "compact", "B": 64, "Hkv": 8, "n": 500, "budget": 500, "share": 0.0, "grown": 1400, "gone": 0.45},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "attn", "draft", "fork", "compact"])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    if op == "attn":
        B, G = _log(rng, 1, 16), rng.randint(1, 8)
        T = _log(rng, 1, min(4096, 2 ** 18 // (B * Hkv * G)))
        most = min(250000, 18 * 10 ** 8 // (B * Hkv * G * T), 8 * 10 ** 6 // (B * Hkv))
        n = 0 if rng.random() < 0.15 else _log(rng, 1, max(1, most - T - 300))
        return {"op": op, "B": B, "Hq": Hkv * G, "Hkv": Hkv, "n": n, "budget": _log(rng, 1, 4096), "share": round(rng.uniform(0.0, 0.9), 2),
                "T": T, "ragged": rng.choice([0.0, 0.5, 1.0]), "grown": rng.choice([0, rng.randint(1, 300)]),
                "layout": rng.choice(["packed", "padded"]), "out": rng.choice(["bf16", "fp32"])}
    c = {"op": op, "Hkv": Hkv, "B": _log(rng, 1 if op == "draft" else 2, 32), "share": round(rng.uniform(0.0, 0.9), 2)}
    c.update(n=_log(rng, 1, 2 ** 20 // (c["B"] * Hkv)), budget=_log(rng, 1, 2048), grown=rng.randint(0, 600))
    if op == "draft":
        c.update(T=_log(rng, 1, 2 ** 17 // (c["B"] * Hkv)), ragged=rng.choice([0.0, 0.5, 1.0]), layout=rng.choice(["packed", "padded"]))
        c["T"] = min(c["T"], 6000)
    elif op == "fork":
        c["keep"] = rng.randint(1, c["B"])
    else:
        c["gone"] = round(rng.uniform(0.05, 0.95), 2)
    return c


# ---------------------------------------------------------------------------------------------- shapes
def _n_new(c):
    """Tokens of every sequence: `ragged` says how much shorter than T they may be, and 1.0 that every third has a single one."""
    T = c["T"]
    out = []
    for b in range(c["B"]):
        t = max(1, T - int(c["ragged"] * (T - 1) * ((b * 7 + 3) % 8) / 8)) if b else T
        out.append(1 if c["ragged"] == 1.0 and b % 3 == 2 else t)
    return out


def _chunk(c):
    """-> (tokens of every sequence, its first token, tokens of the axis)."""
    n_new = _n_new(c)
    if c["layout"] == "padded":
        return n_new, [b * c["T"] for b in range(c["B"])], c["B"] * c["T"]
    return n_new, [sum(n_new[:b]) for b in range(c["B"])], sum(n_new)


def _base(c):
    """Rows of every segment when the prompt had been taken in: a `share` of the heads is short.  Where the lists have grown since, the
    capacities are full and the growth is in pages, one of which every list was given in turn."""
    base, k = [], c["Hkv"]
    short = round(c["share"] * k)
    for b in range(c["B"]):
        n = max(0, c["n"] - (b * 37) % max(1, min(c["n"], 611)))
        if c["op"] == "fork" and not c["grown"] and b >= c["keep"]:
            n = 0  # sequences that have not begun
        for h in range(k):
            rows = min(n, c["budget"]) if (h * 5 + b * 3) % k < short else n
            base.append((rows + ALIGN - 1) // ALIGN * ALIGN if c["grown"] else rows)
    return base


def _lay(c):
    """Segments as a user has them before the call: base rows, capacities, offsets, lengths, pages of every list, the pages' number and a table's width."""
    base = _base(c)
    S = len(base)
    seq = [s // c["Hkv"] for s in range(S)]
    grown = [c["grown"]] * S
    if c["op"] == "attn" and c["grown"]:
        n_new = _n_new(c)
        grown = [c["grown"] + n_new[b] for b in seq]
    elif c["op"] == "attn":
        n_new = _n_new(c)
        base = [x + n_new[b] for x, b in zip(base, seq)]  # the chunk lies in the segments' own rows
    cap = [(x + ALIGN - 1) // ALIGN * ALIGN for x in base]
    off = [sum(cap[:s]) for s in range(S)]
    pages = [(g + PAGE - 1) // PAGE for g in grown]
    lens = [x + g for x, g in zip(base, grown)]
    room = 3 + (c["T"] + PAGE - 1) // PAGE if c["op"] == "draft" else 3
    width = max(pages) + room
    n_pages = S * (max(pages) + room) if c["op"] != "compact" else S * max(pages) + 7
    return {"base": base, "cap": cap, "off": off, "total": sum(cap), "pages": pages, "lens": lens, "width": width, "n_pages": n_pages, "S": S, "seq": seq}


def _table(y):
    """Page p of the lists is given out before page p + 1 of any: [S, width], -1 where there is none."""
    table, at = [[-1] * y["width"] for _ in range(y["S"])], 0
    for p in range(max(y["pages"], default=0)):
        for s in range(y["S"]):
            if p < y["pages"][s]:
                table[s][p] = at
                at += 1
    return table, at


def _parents(c):
    """The first `keep` sequences go on as they are; every other one is replaced by one of them."""
    return [b if b < c["keep"] else (b * 5 + b // 3) % c["keep"] for b in range(c["B"])]


def _gone(c):
    """Sequences that have ended: a share of them, spread over the batch, never the last."""
    return [(b * 61) % 100 < 100 * c["gone"] and b != c["B"] - 1 for b in range(c["B"])]


def work(case):
    c, y = case, _lay(case)
    if c["op"] == "compact":
        table, used = _table(y)
        gone = _gone(c)
        live = [q for s in range(y["S"]) if not gone[y["seq"][s]] for q in table[s] if q >= 0]
        moved = sum(q >= len(live) for q in live)
        return {"bytes": moved * 2 * 2 * PAGE * D * 2 + 8 * len(live), "flops": 0}
    if c["op"] == "fork":
        rows = 0
        for b, p in enumerate(_parents(c)):
            for h in range(c["Hkv"]):
                s = p * c["Hkv"] + h
                over = y["lens"][s] - y["cap"][s]
                rows += 0 if b == p else (over % PAGE if over > 0 else y["lens"][s] % ALIGN)
        return {"bytes": 1024 * rows + 16 * y["S"], "flops": 0}
    n_new = _n_new(c)
    if c["op"] == "draft":
        return {"bytes": 1024 * sum(n_new) * c["Hkv"] + 12 * y["S"], "flops": 0}
    G = c["Hq"] // c["Hkv"]
    seen = sum(n_new[b] * (n - n_new[b]) + n_new[b] * (n_new[b] + 1) // 2 for n, b in zip(y["lens"], y["seq"]))
    io = sum(n_new) * c["Hq"] * (D * (2 + (2 if c["out"] == "bf16" else 4)) + 4)
    return {"bytes": 512 * sum(y["lens"]) + io, "flops": 4 * D * G * seen}


# ---------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    y = _lay(c)
    S, seq = y["S"], y["seq"]
    rows = lambda n: torch.randn(max(n, 1), D, generator=gen, device=dev, dtype=torch.bfloat16)
    k, v, ko, vo = rows(y["total"]), rows(y["total"]), rows(y["n_pages"] * PAGE), rows(y["n_pages"] * PAGE)
    table, used = _table(y)
    st = {"c": c, "y": y}
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    off, cap, lens, tab = ints(y["off"]), ints(y["cap"]), ints(y["lens"]), ints(table)
    # what lies behind a list is no part of it
    row = torch.arange(y["total"], device=dev)
    at = torch.repeat_interleave(torch.arange(S, device=dev), cap.long())
    behind = row - off.long()[at] >= lens.long()[at]
    k[:y["total"]][behind], v[:y["total"]][behind] = float("nan"), float("nan")
    in_page = torch.zeros(y["n_pages"] * PAGE, dtype=torch.bool, device=dev)
    entry = torch.arange(y["width"] * PAGE, device=dev)[None]
    there = entry < (lens - cap).long()[:, None]
    in_page[(tab.long().repeat_interleave(PAGE, 1) * PAGE + entry % PAGE)[there]] = True
    ko[:y["n_pages"] * PAGE][~in_page], vo[:y["n_pages"] * PAGE][~in_page] = float("nan"), float("nan")
    if c["op"] in ("attn", "draft"):
        n_new, start, n_tokens = _chunk(c)
        st["n_new"], st["start"], st["n_tokens"] = n_new, start, n_tokens
    if c["op"] == "attn":
        # a few keys of every list share a direction with its queries and take much of the attention, as they do in a model
        heavy = torch.randn(S, D, generator=gen, device=dev)
        heavy = heavy / heavy.norm(dim=1, keepdim=True) * (2 * D ** 0.25)
        hit = (torch.rand(S, 16, generator=gen, device=dev) * torch.tensor([min(x, m) for x, m in zip(y["base"], y["lens"])], device=dev)[:, None]).long()
        hit = (hit + off.long()[:, None])[torch.tensor(y["base"], device=dev) > 0]
        h16 = heavy[torch.tensor(y["base"], device=dev) > 0].repeat_interleave(16, 0)
        k[hit.reshape(-1)] = (k[hit.reshape(-1)].float() + h16).to(torch.bfloat16)
        # queries, new keys and new values leave a projection side by side: the queries are a strided part of it
        wide = torch.randn(n_tokens, c["Hq"] + 2 * c["Hkv"], D, generator=gen, device=dev)
        owner = torch.repeat_interleave(torch.arange(c["B"], device=dev), torch.tensor([c["T"]] * c["B"] if c["layout"] == "padded" else n_new, device=dev))
        wide[:, :c["Hq"]] += heavy.reshape(c["B"], c["Hkv"], 1, D).expand(-1, -1, c["Hq"] // c["Hkv"], -1).reshape(c["B"], c["Hq"], D)[owner]
        st["q"] = wide.to(torch.bfloat16)[:, :c["Hq"]]
        st["out"] = torch.full((n_tokens, c["Hq"], D), 0.015625, device=dev, dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32)
        st["lse"] = torch.full((n_tokens, c["Hq"]), 7.0, device=dev)
    if c["op"] == "draft":
        st["kn"], st["vn"] = (rows(n_tokens * 2 * c["Hkv"]).reshape(n_tokens, 2 * c["Hkv"], D)[:, i * c["Hkv"]:(i + 1) * c["Hkv"]] for i in range(2))
    t = {"k": k, "v": v, "ko": ko, "vo": vo, "off": off, "cap": cap, "len": lens, "table": tab}
    st["held"] = torch.tensor(y["pages"], device=dev)
    if c["op"] == "compact":
        keep = torch.tensor([0 if _gone(c)[b] else 1 for b in seq], device=dev)
        st["held"] = st["held"] * keep
        t["len"] = lens * keep.int()
    st["table0"] = t["table"].clone()
    if own:
        import numpy as np
        import paper_2608_30295_b200 as ck
        cache = ck.Cache(c["B"], c["Hkv"], y["base"], 0, dev)
        pages = cache.attach_pages(y["n_pages"], y["width"])
        pages.table[:] = table
        pages.table_dev.copy_(tab)
        pages.seg_pages[:] = y["pages"]
        pages.struct.next_free = used
        cache.k_pool.copy_(k), cache.v_pool.copy_(v)
        pages.k_ovf.copy_(ko), pages.v_ovf.copy_(vo)
        cache.set_lengths(y["lens"])
        if c["op"] == "compact":
            ck.catekv_truncate(cache, np.array([1 << 30 if g else 0 for g in _gone(c)], dtype=np.int32))
            st["host0"] = (pages.table.copy(), pages.struct.next_free, pages.struct.released)
        t.update(k=cache.k_pool, v=cache.v_pool, ko=pages.k_ovf, vo=pages.v_ovf, off=cache.seg_off_dev, cap=cache.seg_cap_dev,
                 len=cache.seg_len_dev, table=pages.table_dev)
        st.update(ck=ck, cache=cache, pages=pages)
        if c["op"] in ("attn", "draft"):
            st["chunk"] = ck.Chunk(n_new, start, n_tokens)
        if c["op"] == "attn":
            st["ws"] = ck.chunk_attn_workspace(cache, st["chunk"], c["Hq"])
        if c["op"] == "draft":
            st["drop"] = np.array(n_new, dtype=np.int32)
        if c["op"] == "fork":
            st["parent"] = np.array(_parents(c), dtype=np.int32)
    elif c["op"] in ("attn", "draft"):
        st["per_seg"] = torch.tensor(n_new, device=dev)[torch.tensor(seq, device=dev)]
        st["first"] = torch.tensor(start, device=dev)[torch.tensor(seq, device=dev)]
    elif c["op"] == "fork":
        parent = torch.tensor(_parents(c), device=dev)[torch.tensor(seq, device=dev)] * c["Hkv"] + torch.arange(S, device=dev) % c["Hkv"]
        st["from"] = parent
    st["t"] = t
    return st


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    op = state["c"]["op"]
    return {"attn": _run_attn, "draft": _run_draft, "fork": _run_fork, "compact": _run_compact}[op](state, state["c"], state["t"])


def _places(t, row):
    """Of rows `row` [S, n] of every segment: the rows of the pools, the rows of the overflow pools, and which of the two."""
    o = row - t["cap"].long()[:, None]
    page = torch.gather(t["table"].long(), 1, (o // PAGE).clamp(min=0, max=t["table"].shape[1] - 1))
    return t["off"].long()[:, None] + row, (page * PAGE + o % PAGE).clamp(min=0), o >= 0


def _run_attn(st, c, t):
    if own:
        st["ck"].catekv_chunk_attn(st["cache"], st["chunk"], st["q"], st["out"], st["lse"], ws=st["ws"])
        return [st["out"], st["lse"]]
    S, G, L, T = t["len"].numel(), c["Hq"] // c["Hkv"], max(st["y"]["lens"]), max(st["n_new"])
    row = torch.arange(L, device="cuda")[None].expand(S, -1)
    there = row < t["len"][:, None]
    in_pool, in_page, paged = _places(t, row)
    kv = []
    for x in ("k", "v"):
        z = t[x][torch.where(there & ~paged, in_pool, 0)].float()
        if c["grown"]:
            z[there & paged] = t[x + "o"][in_page[there & paged]].float()
        kv.append(z.masked_fill_(~there[..., None], 0.0))
    i = torch.arange(T, device="cuda")
    asked = i[None] < st["per_seg"][:, None]  # [S, T]: the segment has a query there
    token = (st["first"][:, None] + i[None]).clamp(max=st["n_tokens"] - 1)
    head = (torch.arange(S, device="cuda") % c["Hkv"] * G)[:, None, None] + torch.arange(G, device="cuda")[None, None]
    q = st["q"][token[..., None], head].float().reshape(S, T * G, D)
    sees = t["len"].long()[:, None] - st["per_seg"][:, None] + i[None] + 1  # [S, T]
    x = torch.matmul(q, kv[0].transpose(1, 2)).div_(math.sqrt(D))
    x.masked_fill_(row[:, None] >= sees.repeat_interleave(G, 1)[..., None], float("-inf"))
    m = x.amax(dim=2, keepdim=True)
    x.sub_(torch.where(m > float("-inf"), m, 0.0)).exp_()
    s = x.sum(dim=2, keepdim=True)
    o = torch.matmul(x, kv[1]) / torch.where(s > 0, s, 1.0)
    lse = (m + torch.log(s)).squeeze(2)
    to, at = token[..., None].expand(-1, -1, G)[asked], head.expand(-1, T, -1)[asked]
    st["out"][to, at] = o.reshape(S, T, G, D)[asked].to(st["out"].dtype)
    st["lse"][to, at] = lse.reshape(S, T, G)[asked]
    return [st["out"], st["lse"]]


def _given(t, held, n):
    """Pages for `n` [S] more of every list, which holds `held`: the lowest free ones, in the order of the lists; their table entries."""
    slot = torch.arange(t["table"].shape[1], device="cuda")[None]
    free = torch.ones(t["ko"].shape[0] // PAGE, dtype=torch.bool, device="cuda")
    free[t["table"][slot < held[:, None]].long()] = False
    free = torch.nonzero(free).squeeze(1).int()
    want = (slot >= held[:, None]) & (slot < (held + n)[:, None])
    t["table"][want] = free[: int(n.sum())]
    return want


def _run_draft(st, c, t):
    if own:
        ck, cache = st["ck"], st["cache"]
        ck.catekv_pages_reserve(cache, c["T"])
        ck.catekv_append_chunk(cache, st["chunk"], st["kn"], st["vn"])
        ck.catekv_truncate(cache, st["drop"])
    else:
        S, T = t["len"].numel(), max(st["n_new"])
        n = t["len"].long()
        need = ((n + c["T"] - t["cap"].long()).clamp(min=0) + PAGE - 1) // PAGE
        _given(t, st["held"], (need - st["held"]).clamp(min=0))
        i = torch.arange(T, device="cuda")[None]
        new = i < st["per_seg"][:, None]
        in_pool, in_page, paged = _places(t, n[:, None] + i)
        token = (st["first"][:, None] + i)
        head = (torch.arange(S, device="cuda") % c["Hkv"])[:, None].expand(-1, T)
        for x, z in (("k", st["kn"]), ("v", st["vn"])):
            a, b = new & ~paged, new & paged
            t[x][in_pool[a]] = z[token[a], head[a]]
            t[x + "o"][in_page[b]] = z[token[b], head[b]]
        t["len"].add_(st["per_seg"].int()).sub_(st["per_seg"].int())
    return [t[x] for x in ("k", "v", "ko", "vo", "len", "table")]


def _run_fork(st, c, t):
    if own:
        st["ck"].catekv_fork(st["cache"], st["parent"])
    else:
        S, p = t["len"].numel(), st["from"]
        new = p != torch.arange(S, device="cuda")
        n, cap, held = t["len"].long()[p], t["cap"].long()[p], st["held"][p]
        flat = n <= cap  # nothing in pages: the rows from the last multiple of 128 on are copied to pages
        base = torch.where(flat, n // ALIGN * ALIGN, cap)
        full = torch.where(flat, 0, (n - base) // PAGE)
        rest = n - base - full * PAGE
        in_pool, in_page, paged = _places(t, (n - rest)[:, None] + torch.zeros(1, ALIGN, dtype=torch.long, device="cuda"))
        row = (n - rest)[:, None] + torch.arange(ALIGN, device="cuda")[None]
        old = {x: t[x].clone() for x in ("off", "cap", "len", "table")}
        par = {x: old[x][p] for x in old}
        in_pool, in_page, paged = _places(par, row)
        slot = torch.arange(t["table"].shape[1], device="cuda")[None]
        t["table"].copy_(torch.where(new[:, None] & (slot < full[:, None]), par["table"], t["table"]))
        held = torch.where(new, full, st["held"])
        more = torch.where(new, (rest + PAGE - 1) // PAGE, 0)
        _given(t, held, more)
        st["held"] = held + more
        for x, z in (("off", p), ("len", p)):
            t[x].copy_(old[x][z])
        t["cap"].copy_(torch.where(new, base, old["cap"].long()).int())
        copied = new[:, None] & (torch.arange(ALIGN, device="cuda")[None] < rest[:, None])
        _, to, _ = _places(t, row)
        for x in ("k", "v"):
            z = torch.where(paged[..., None], t[x + "o"][in_page.clamp(max=t["ko"].shape[0] - 1)], t[x][in_pool.clamp(max=t["k"].shape[0] - 1)])
            t[x + "o"][to[copied]] = z[copied]
    return [t[x] for x in ("ko", "vo", "off", "cap", "len", "table")]


def _run_compact(st, c, t):
    t["table"].copy_(st["table0"])  # back to where the pages lie scattered, so that it can be run again (they are still there)
    if own:
        table, next_free, released = st["host0"]
        st["pages"].table[:] = table
        st["pages"].struct.next_free, st["pages"].struct.released = next_free, released
        st["ck"].catekv_pages_compact(st["cache"])
    else:
        held = torch.arange(t["table"].shape[1], device="cuda")[None] < st["held"][:, None]
        used = torch.zeros(t["ko"].shape[0] // PAGE, dtype=torch.bool, device="cuda")
        used[t["table"][held].long()] = True
        live = used.sum()
        page = torch.arange(used.numel(), device="cuda")
        src, dst = torch.nonzero(used & (page >= live)).squeeze(1), torch.nonzero(~used & (page < live)).squeeze(1)
        for x in ("ko", "vo"):
            z = t[x].reshape(-1, PAGE * D)
            z[dst] = z[src]
        page[src] = dst
        t["table"].copy_(torch.where(held, page[t["table"].long().clamp(min=0)].int(), t["table"]))
    return [t["ko"], t["vo"], t["table"]]


# ---------------------------------------------------------------------------------------------- in 64 bits
def _rows64(st, name, s, n):
    """The first n rows of list s, from the tables of the case."""
    y, t = st["y"], st["t"]
    base = min(n, y["cap"][s])
    parts = [t[name][y["off"][s]:y["off"][s] + base].double()]
    if n > base:
        pages = st["table0"][s, : (n - base + PAGE - 1) // PAGE].long()
        parts.append(t[name + "o"].reshape(-1, PAGE, D)[pages].reshape(-1, D)[: n - base].double())
    return torch.cat(parts)


def exact(case, seed):
    c = case
    if c["op"] != "attn":
        # rows are copied as they are: the outputs are the inputs at other places, which whole tables of integers say
        return None
    st = prepare(case, seed)
    y, G = st["y"], c["Hq"] // c["Hkv"]
    out, lse = st["out"].double(), st["lse"].double()
    for s, n in enumerate(y["lens"]):
        b, h = divmod(s, c["Hkv"])
        m, t0 = st["n_new"][b], st["start"][b]
        k, v = _rows64(st, "k", s, n), _rows64(st, "v", s, n)
        step = max(1, 2 ** 27 // max(n, 1))
        for g in range(G):
            for i in range(0, m, step):
                e = min(m, i + step)
                x = st["q"][t0 + i:t0 + e, h * G + g].double() @ k.T / math.sqrt(D)
                if e > 1 or i:
                    last = torch.arange(i, e, device="cuda") + n - m
                    x.masked_fill_(torch.arange(n, device="cuda")[None] > last[:, None], float("-inf"))
                z = torch.logsumexp(x, dim=1)
                lse[t0 + i:t0 + e, h * G + g] = z
                out[t0 + i:t0 + e, h * G + g] = torch.exp(x - z[:, None]) @ v
    return [out, lse]
