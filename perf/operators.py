"""Exact attention and the key/value cache that serves it, as cases that can be prepared, run and priced.

Four operators: `prompt` (attention over packed sequences), `store` (keys and values of new tokens into a paged 8-bit
cache), `attend` (attention over that cache, with the weight that every cached token received) and `evict` (the cache
cut down to a budget by those weights).  With `own` false `run` computes them from elementary torch operations in 32
bits, with `own` true by the library's calls; `exact` computes them in 64 bits from their definitions.

Cache layout: K codes [pages, Hkv, page, d], V codes [pages, Hkv, d, page] (e4m3), one power-of-two scale per block (page,
head) of each; a sequence's pages are a row of `table`, its tokens the first lengths[b] slots of them; W [B, Hkv, slots]
the weight that each slot has received.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
_TDTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn


def listed():
    return [
        # one head over 256 tokens in float: the smallest prompt anyone runs, launches and latency
        _prompt("prompt_tiny_f32", 1, 1, 1, 64, 256, 256, 0, "f32", 1),
        # an image with its caption, every token sees every other
        _prompt("prompt_image_text", 8, 12, 1, 64, 274, 274, 0, "bf16", 0),
        # one clip in float
        _prompt("prompt_clip_f32", 1, 12, 1, 64, 1600, 1600, 0, "f32", 1),
        # a batch of prompts of very different lengths, packed, four query heads to a key head
        _prompt("prompt_packed", 8, 8, 4, 128, 257, 4096, 0, "bf16", 1),
        # a long video, the largest prompt: 16384 tokens, 16 heads
        _prompt("prompt_long_video", 1, 4, 4, 128, 16384, 16384, 0, "bf16", 1),
        # one decode step's tokens of 64 sequences
        _store("store_step", 64, 8, 128, 64, 1, 1, 200, 4000, "bf16"),
        # prompts of a batch, the first of them a few tokens behind a cached beginning
        _store("store_prompts", 8, 8, 128, 64, 257, 4096, 0, 100, "bf16"),
        # one short conversation: latency
        _attend("attend_single", 1, 2, 4, 64, 64, 300, 300, 1, 0, "bf16"),
        # a batch of conversations in decode, weights collected for a later eviction
        _attend("attend_batch", 32, 8, 4, 128, 64, 700, 8100, 1, 1, "bf16"),
        # one very long context
        _attend("attend_long", 1, 8, 4, 128, 64, 131072, 131072, 1, 0, "bf16"),
        # one conversation a little over its budget
        _evict("evict_single", 1, 2, 64, 64, 1100, 1100, 1024, 64),
        # a batch of long ones cut in half
        _evict("evict_batch", 16, 8, 128, 64, 6000, 8190, 4096, 512),
    ]


def _prompt(name, B, Hkv, G, d, shortest, longest, queries, dtype, causal):
    """`queries`: rows of Q per sequence, 0: as many as of K."""
    return _named(name, dict(op="prompt", B=B, Hkv=Hkv, G=G, d=d, shortest=shortest, longest=longest, queries=queries,
                             dtype=dtype, causal=causal))


def _store(name, B, Hkv, d, page, shortest, longest, before_least, before_most, dtype):
    """New tokens per sequence from `shortest` to `longest`, behind before_least .. before_most cached ones."""
    return _named(name, dict(op="store", B=B, Hkv=Hkv, G=1, d=d, page=page, shortest=shortest, longest=longest,
                             before_least=before_least, before_most=before_most, dtype=dtype))


def _attend(name, B, Hkv, G, d, page, shortest, longest, queries, weights, dtype):
    return _named(name, dict(op="attend", B=B, Hkv=Hkv, G=G, d=d, page=page, shortest=shortest, longest=longest,
                             queries=queries, weights=weights, dtype=dtype))


def _evict(name, B, Hkv, d, page, shortest, longest, budget, recent):
    return _named(name, dict(op="evict", B=B, Hkv=Hkv, G=1, d=d, page=page, shortest=shortest, longest=longest,
                             budget=budget, recent=recent, dtype="bf16"))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    while True:
        op = rng.choices(["prompt", "store", "attend", "evict"], [5, 3, 5, 3])[0]
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        Hkv, G = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 4, 8])
        page = rng.choice([16, 32, 64, 64, 128])
        if op == "prompt":
            d = rng.choice([64, 64, 128, 128, 80, 96, 256])
            B = rng.choice([1, 1, 2, 4, 8, 16])
            longest = _log(rng, 16, 16384)
            shortest = max(1, int(longest * rng.random()))
            queries = _log(rng, 1, longest) if rng.random() < 0.3 else 0
            c = _prompt(None, B, Hkv, G, d, shortest, longest, queries, dtype, int(rng.random() < 0.7))
            if B * Hkv * G * (queries or longest) * longest <= 4.0e9 and work(c)["flops"] <= (1.1e12 if dtype == "bf16" else 8e10) and work(c)["flops"] >= 1e6:
                return c
            continue
        d = rng.choice([64, 64, 128, 128, 80, 96, 256])
        B = _log(rng, 1, 64)
        if op == "store":
            longest = 1 if rng.random() < 0.4 else _log(rng, 2, 8192)
            shortest = max(1, int(longest * rng.random()))
            before = _log(rng, 1, 4096)
            c = _store(None, B, Hkv, d, page, shortest, longest, before // 3, before, dtype)
            if sum(_lens(c)) * Hkv * d <= 1.8e7 and B * (before + longest) * Hkv * d <= 2e8:
                return c
        elif op == "attend":
            longest = _log(rng, 32, 131072)
            shortest = max(1, int(longest * rng.random()))
            queries = 1 if rng.random() < 0.7 else rng.randint(2, 8)
            c = _attend(None, B, Hkv, G, d, page, max(shortest, queries), max(longest, queries), queries, int(rng.random() < 0.4), dtype)
            if B * longest * Hkv * d <= 2e8 and sum(_lens(c)) * Hkv * (2 * d + 8 * G * queries) <= 3e8:
                return c
        else:
            longest = _log(rng, 64, 32768)
            shortest = max(1, int(longest * rng.uniform(0.3, 1.0)))
            budget = max(1, int(longest * rng.uniform(0.2, 0.95)))
            c = _evict(None, B, Hkv, d, page, shortest, longest, budget, rng.randint(0, budget))
            if B * longest * Hkv * d <= 1.3e8:
                return c


def _spread(a, b, B):
    """B whole numbers between a and b, both among them, in no order."""
    f = [(i * 0.6180339887498949) % 1.0 for i in range(B)]
    lo, hi = min(f), max(f)
    return [b if B == 1 else int(round(a + (b - a) * (v - lo) / (hi - lo))) for v in f]


def _lens(c):
    return _spread(c["shortest"], c["longest"], c["B"])


def _q_lens(c):
    return [c["queries"] or n for n in _lens(c)] if c["op"] == "prompt" else [c["queries"]] * c["B"]


def _before(c):
    return _spread(c["before_least"], c["before_most"], c["B"])[::-1]


def _pages(n, page):
    return (n + page - 1) // page


def _offsets(lens):
    o = [0]
    for n in lens:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device=DEV)


def _tokens(g, rows, heads, d, t):
    """Rows of an attention head: some features larger than others, a part that the tokens share."""
    x = torch.randn(rows, heads, d, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(1, heads, d, generator=g, device=DEV))
    return (x + 0.5 * torch.randn(1, heads, d, generator=g, device=DEV)).to(t)


def _queries(g, rows, heads, d, t):
    """Queries that make scores of a spread of two or three: some keys stand out, none is alone."""
    return (2.0 * torch.randn(rows, heads, d, generator=g, device=DEV)).to(t)


def _pool(g, c, tables):
    """A pool of codes and scales, and `tables` page tables of B rows without a common page: lists of pages per sequence."""
    Hkv, d, page = c["Hkv"], c["d"], c["page"]
    pages = sum(sum(t) for t in tables) + 3
    order = torch.randperm(pages, generator=g, device=DEV).int()
    s = {}
    for name, shape in (("K", (pages, Hkv, page, d)), ("V", (pages, Hkv, d, page))):
        code = torch.empty(shape, dtype=F8, device=DEV)
        for at in range(0, pages, 4096):      # (in parts: 32 bits of every slot at once are four times the pool)
            part = code[at:at + 4096]
            part.copy_((torch.randn(part.shape, generator=g, device=DEV) * 100.0).clamp_(-448, 448))
        s[name] = code
        s[name + "s"] = torch.exp2(torch.randint(-8, -5, (pages, Hkv), generator=g, device=DEV).float())
    out, at = [], 0
    for need in tables:
        most = max(need)
        rows = torch.full((c["B"], most), -1, dtype=torch.int32, device=DEV)      # what no token needs names no page
        for b, n in enumerate(need):
            rows[b, :n] = order[at:at + n]
            at += n
        out.append(rows)
    return s, out


def prepare(case, seed):
    c = dict(case)
    op, B, Hkv, G, d, t = c["op"], c["B"], c["Hkv"], c["G"], c["d"], _TDTYPE[c["dtype"]]
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    Hq = Hkv * G
    lens = _lens(c)
    s = dict(case=c, op=op)
    if op == "prompt":
        ql = _q_lens(c)
        nq, nk = sum(ql), sum(lens)
        s.update(Q=_queries(g, nq, Hq, d, t), K=_tokens(g, nk, Hkv, d, t), V=_tokens(g, nk, Hkv, d, t), q_off=_offsets(ql),
                 k_off=_offsets(lens), O=torch.zeros(nq, Hq, d, dtype=t, device=DEV), lse=torch.zeros(Hq, nq, device=DEV),
                 scale=1.0 / math.sqrt(d))
        if own:
            import paper_2507_02957_amd as csat
            s["dims"] = csat.make_packed_dims(B, Hq, Hkv, d, nq, nk, max(ql), max(lens), c["dtype"], causal=bool(c["causal"]))
            s["ws"] = torch.empty(csat.csat_prompt_workspace_bytes(s["dims"]), dtype=torch.uint8, device=DEV)
        return s
    page = c["page"]
    if op == "store":
        before = _before(c)
        total = [n + m for n, m in zip(before, lens)]
        pool, (table,) = _pool(g, c, [[_pages(n, page) for n in total]])
        s.update(pool, table=table, lengths=torch.tensor(total, dtype=torch.int32, device=DEV), k_off=_offsets(lens),
                 Kn=_tokens(g, sum(lens), Hkv, d, t), Vn=_tokens(g, sum(lens), Hkv, d, t))
        if own:
            import paper_2507_02957_amd as csat
            s["dims"] = csat.make_packed_dims(B, Hkv, Hkv, d, sum(lens), sum(lens), max(lens), max(lens), c["dtype"])
            s["cache"] = csat.make_cache(s["K"], s["V"], s["Ks"], s["Vs"], table, s["lengths"], max(total))
        return s
    if op == "attend":
        pool, (table,) = _pool(g, c, [[_pages(n, page) for n in lens]])
        ql = _q_lens(c)
        nq = sum(ql)
        s.update(pool, table=table, lengths=torch.tensor(lens, dtype=torch.int32, device=DEV), q_off=_offsets(ql),
                 Q=_queries(g, nq, Hq, d, t), O=torch.zeros(nq, Hq, d, dtype=t, device=DEV), lse=torch.zeros(Hq, nq, device=DEV),
                 W=torch.zeros(B, Hkv, table.shape[1] * page, device=DEV) if c["weights"] else None, scale=1.0 / math.sqrt(d))
        if own:
            import paper_2507_02957_amd as csat
            s["dims"] = csat.make_packed_dims(B, Hq, Hkv, d, nq, nq, max(ql), max(ql), c["dtype"], causal=True)
            s["cache"] = csat.make_cache(s["K"], s["V"], s["Ks"], s["Vs"], table, s["lengths"], max(lens))
            s["ws"] = torch.empty(csat.csat_cache_workspace_bytes(s["dims"], s["cache"]), dtype=torch.uint8, device=DEV)
        return s
    budget = c["budget"]
    keep = [min(n, budget) for n in lens]
    pool, (table, to) = _pool(g, c, [[_pages(n, page) for n in lens], [_pages(n, page) for n in keep]])
    W = torch.exp(2.0 * torch.randn(B, Hkv, table.shape[1] * page, generator=g, device=DEV))
    W *= (torch.rand(W.shape, generator=g, device=DEV) > 0.1)      # one token in ten that nothing has looked at: ties
    s.update(pool, table=table, lengths=torch.tensor(lens, dtype=torch.int32, device=DEV), W=W, to=to,
             W_to=torch.zeros(B, Hkv, to.shape[1] * page, device=DEV), kept=torch.zeros(B, Hkv, budget, dtype=torch.int32, device=DEV),
             lengths_to=torch.zeros(B, dtype=torch.int32, device=DEV))
    if own:
        import paper_2507_02957_amd as csat
        s["dims"] = csat.make_packed_dims(B, Hkv, Hkv, d, B, B, 1, 1, c["dtype"])
        s["from"] = csat.make_cache(s["K"], s["V"], s["Ks"], s["Vs"], table, s["lengths"], max(lens))
        s["to_cache"] = csat.make_cache(s["K"], s["V"], s["Ks"], s["Vs"], to, s["lengths_to"], max(keep))
    return s


def run(s):
    op = s["op"]
    if own:
        import paper_2507_02957_amd as csat
        if op == "prompt":
            csat.csat_prompt_attention(s["dims"], s["Q"], s["K"], s["V"], s["q_off"], s["k_off"], s["scale"], s["O"], s["lse"], s["ws"])
            return s["O"], s["lse"]
        if op == "store":
            csat.csat_cache_store(s["dims"], s["cache"], s["Kn"], s["Vn"], s["k_off"])
            return s["K"], s["V"], s["Ks"], s["Vs"]
        if op == "attend":
            csat.csat_cache_attention(s["dims"], s["cache"], s["Q"], s["q_off"], s["scale"], 0.0, s["O"], s["lse"], s["W"], s["ws"])
            return s["O"], s["lse"], s["W"]
        csat.csat_cache_evict(s["dims"], s["from"], s["to_cache"], s["W"], s["W_to"], s["case"]["budget"], s["case"]["recent"], s["kept"])
        return s["K"], s["V"], s["Ks"], s["Vs"], s["W_to"], s["kept"], s["lengths_to"]
    return {"prompt": _plain_prompt, "store": _plain_store, "attend": _plain_attend, "evict": _plain_evict}[op](s)


# ---- the plain forms: elementary operations in 32 bits, sequences padded to the longest


def _rows_of(off, rows, longest):
    """Of packed rows: each row's sequence and place, and the rows of each sequence, padded, with whether they exist."""
    at = torch.arange(rows, device=DEV)
    seq = torch.bucketize(at, off[1:].long(), right=True)
    place = at - off.long()[seq]
    i = torch.arange(longest, device=DEV)
    there = i < (off[1:] - off[:-1]).long()[:, None]
    return seq, place, torch.where(there, off[:-1].long()[:, None] + i, 0), there


def _plain_softmax(S, visible):
    """Weights and log-sum-exp over the last axis; rows that see nothing: 0 and -inf."""
    S = torch.where(visible, S, -math.inf)
    m = S.amax(-1, keepdim=True)
    m0 = torch.where(m == -math.inf, 0.0, m)
    P = torch.exp(S - m0)
    l = P.sum(-1, keepdim=True)
    P = P / torch.where(l == 0, 1.0, l)
    return P, (m0 + torch.log(l)).squeeze(-1)


def _plain_prompt(s):
    c = s["case"]
    B, Hkv, G, d = c["B"], c["Hkv"], c["G"], c["d"]
    mq, mk = c["queries"] or c["longest"], c["longest"]
    nq = s["Q"].shape[0]
    qs, qp, qi, _ = _rows_of(s["q_off"], nq, mq)
    _, _, ki, kt = _rows_of(s["k_off"], s["K"].shape[0], mk)
    Q = s["Q"].float()[qi].view(B, mq, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * mq, d)
    K = s["K"].float()[ki].permute(0, 2, 3, 1).reshape(B * Hkv, d, mk)
    V = s["V"].float()[ki].permute(0, 2, 1, 3).reshape(B * Hkv, mk, d)
    S = torch.bmm(Q, K).view(B, Hkv, G, mq, mk) * s["scale"]
    visible = kt[:, None, :]
    if c["causal"]:
        nk, n = (s["k_off"][1:] - s["k_off"][:-1]).long(), (s["q_off"][1:] - s["q_off"][:-1]).long()
        last = torch.arange(mq, device=DEV)[None, :] + (nk - n)[:, None]
        visible = visible & (torch.arange(mk, device=DEV) <= last[:, :, None])
    P, lse = _plain_softmax(S, visible.view(B, 1, 1, -1, mk))
    O = torch.bmm(P.view(B * Hkv, G * mq, mk), V).view(B, Hkv * G, mq, d)
    s["O"].copy_(O[qs, :, qp])
    s["lse"].copy_(lse.reshape(B, Hkv * G, mq)[qs, :, qp].t())
    return s["O"], s["lse"]


def _plain_scale(amax):
    """Smallest power of two with amax <= 448 of it."""
    f, e = torch.frexp(amax)
    e = torch.where(amax == 0, -118, torch.where(f <= 0.875, e - 9, e - 8)).clamp(min=-118)
    return ((e + 127) << 23).int().view(torch.float32)      # (2^e by its bits: a power function may miss it by a rounding)


def _plain_block(new, old_code, old_scale, is_new, is_old):
    """Codes and scale of blocks [.., slots, d] from new values and old codes; masks [.., slots, 1]."""
    amax = torch.where(is_new & torch.isfinite(new), new.abs(), 0.0).amax((-1, -2))
    scale = _plain_scale(amax)
    scale = torch.where(is_old.any(-2).squeeze(-1), torch.maximum(scale, old_scale), scale)
    quantised = (new / scale[..., None, None]).to(F8)
    moved = (old_code.view(F8).float() * (old_scale / scale)[..., None, None]).to(F8)
    code = torch.where(is_new, quantised.view(torch.uint8), torch.where(is_old, moved.view(torch.uint8), old_code))
    return code, scale


def _plain_store(s):
    c = s["case"]
    B, Hkv, d, page = c["B"], c["Hkv"], c["d"], c["page"]
    rows = s["Kn"].shape[0]
    seq, place, _, _ = _rows_of(s["k_off"], rows, 1)
    new = (s["k_off"][1:] - s["k_off"][:-1]).long()
    total = s["lengths"].long()
    start = total - new
    first = start // page
    T = _pages(c["longest"] - 1, page) + 1                      # pages that a sequence's new tokens may reach
    slot = (start - first * page)[seq] + place                  # of each new row, from its sequence's first page on
    i = first[:, None] + torch.arange(T, device=DEV)
    used = i * page < total[:, None]
    ids = torch.gather(s["table"].long(), 1, i.clamp(max=s["table"].shape[1] - 1))
    spare = s["K"].shape[0]                                     # (a page of nobody, for those that are not there)
    ids = torch.where(used, ids, spare)
    at = i[:, :, None] * page + torch.arange(page, device=DEV)
    is_old = (at < start[:, None, None])[:, :, None, :, None]
    is_new = ((at >= start[:, None, None]) & (at < total[:, None, None]))[:, :, None, :, None]
    for name, x in (("K", s["Kn"]), ("V", s["Vn"])):
        pool, scales = s[name], s[name + "s"]
        codes = torch.cat([pool.view(torch.uint8), torch.zeros_like(pool[:1]).view(torch.uint8)])
        both = torch.cat([scales, torch.ones_like(scales[:1])])
        value = torch.zeros(B, T * page, Hkv, d, device=DEV)
        value[seq, slot] = x.float()
        value = value.view(B, T, page, Hkv, d).transpose(2, 3)
        old = codes[ids]
        old = old if name == "K" else old.transpose(-1, -2)
        code, scale = _plain_block(value, old, both[ids], is_new, is_old)
        codes[ids] = code if name == "K" else code.transpose(-1, -2)
        both[ids] = scale
        pool.view(torch.uint8).copy_(codes[:spare])
        scales.copy_(both[:spare])
    return s["K"], s["V"], s["Ks"], s["Vs"]


def _plain_cached(s, name, table):
    """Values of the cached tokens, [B, Hkv, slots, d] in 32 bits."""
    ids = table.long().clamp(min=0)
    x = s[name][ids] if s[name].dtype != F8 else s[name].view(torch.uint8)[ids].view(F8)
    x = x.float() * s[name + "s"][ids][..., None, None]
    x = x if name == "K" else x.transpose(-1, -2)
    B, n, Hkv, page, d = x.shape
    return x.transpose(1, 2).reshape(B, Hkv, n * page, d)


def _plain_attend(s):
    c = s["case"]
    B, Hkv, G, d, n = c["B"], c["Hkv"], c["G"], c["d"], c["queries"]
    K, V = _plain_cached(s, "K", s["table"]), _plain_cached(s, "V", s["table"])
    slots = K.shape[2]
    Q = s["Q"].float().view(B, n, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * n, d)
    S = torch.bmm(Q, K.view(B * Hkv, slots, d).transpose(1, 2).contiguous()).view(B, Hkv, G, n, slots) * s["scale"]
    last = s["lengths"].long()[:, None] - n + torch.arange(n, device=DEV)
    visible = torch.arange(slots, device=DEV) <= last[:, :, None]
    visible = visible.view(B, 1, 1, n, slots)
    P, lse = _plain_softmax(S, visible)
    there = torch.arange(slots, device=DEV)[None, None, :, None] < s["lengths"].long()[:, None, None, None]
    V = torch.where(there, V, 0.0)
    O = torch.bmm(P.view(B * Hkv, G * n, slots), V.view(B * Hkv, slots, d)).view(B, Hkv * G, n, d)
    s["O"].copy_(O.transpose(1, 2).reshape(B * n, Hkv * G, d))
    s["lse"].copy_(lse.reshape(B, Hkv * G, n).transpose(0, 1).reshape(Hkv * G, B * n))
    if s["W"] is not None:
        s["W"].copy_(torch.where(there.squeeze(-1), P.sum((2, 3)), s["W"]))
    return s["O"], s["lse"], s["W"]


def _plain_evict(s):
    c = s["case"]
    B, Hkv, d, page, budget = c["B"], c["Hkv"], c["d"], c["page"], c["budget"]
    L = s["lengths"].long()
    keep = L.clamp(max=budget)
    recent = keep.clamp(max=c["recent"])
    slots = s["table"].shape[1] * page
    i = torch.arange(slots, device=DEV)
    old = (i < (L - recent)[:, None])[:, None, :]
    late = ((i >= (L - recent)[:, None]) & (i < L[:, None]))[:, None, :]
    key = torch.where(late, math.inf, torch.where(old, s["W"], -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    width = s["to"].shape[1] * page
    chosen = torch.where(torch.arange(slots, device=DEV) < keep[:, None, None], order, slots)
    chosen = torch.sort(chosen, dim=-1)[0]
    chosen = torch.nn.functional.pad(chosen, (0, max(0, width - slots)), value=slots)[..., :width]
    there = chosen < slots
    at = torch.where(there, chosen, 0)
    s["kept"].copy_(torch.where(there, chosen, -1)[..., :budget] if budget <= width else
                    torch.nn.functional.pad(torch.where(there, chosen, -1), (0, budget - width), value=-1))
    s["lengths_to"].copy_(keep)
    s["W_to"].copy_(torch.where(there, torch.gather(s["W"], 2, at), s["W_to"]))
    n = s["to"].shape[1]
    used = torch.arange(n, device=DEV) * page < keep[:, None]
    spare = s["K"].shape[0]
    ids = torch.where(used, s["to"].long(), spare)
    is_new = there.view(B, Hkv, n, page).transpose(1, 2)[..., None]
    for name in ("K", "V"):
        pool, scales = s[name], s[name + "s"]
        value = torch.gather(_plain_cached(s, name, s["table"]), 2, at[..., None].expand(-1, -1, -1, d))
        value = value.view(B, Hkv, n, page, d).transpose(1, 2)
        codes = torch.cat([pool.view(torch.uint8), torch.zeros_like(pool[:1]).view(torch.uint8)])
        both = torch.cat([scales, torch.ones_like(scales[:1])])
        was = codes[ids] if name == "K" else codes[ids].transpose(-1, -2)
        code, scale = _plain_block(value, was, both[ids], is_new, torch.zeros_like(is_new))
        codes[ids] = code if name == "K" else code.transpose(-1, -2)
        both[ids] = scale
        pool.view(torch.uint8).copy_(codes[:spare])
        scales.copy_(both[:spare])
    return s["K"], s["V"], s["Ks"], s["Vs"], s["W_to"], s["kept"], s["lengths_to"]


# ---- what a pass cannot do without


def work(case):
    c = case
    op, B, Hkv, G, d = c["op"], c["B"], c["Hkv"], c["G"], c["d"]
    e = 4 if c["dtype"] == "f32" else 2
    Hq, lens = Hkv * G, _lens(c)
    if op in ("prompt", "attend"):
        pairs, nq = 0, 0
        for n, q in zip(lens, _q_lens(c)):
            nq += q
            if op == "prompt" and not c["causal"]:
                pairs += q * n
            else:      # row i of q sees n - q + 1 + i keys, where that is positive
                see = min(q, n)
                pairs += see * n - see * (see - 1) // 2
        rows = nq * Hq * (2 * d * e + 4)
        flops = 4.0 * d * Hq * pairs
        if op == "prompt":
            return {"bytes": float(rows + 2 * sum(lens) * Hkv * d * e), "flops": flops}
        blocks = sum(_pages(n, c["page"]) for n in lens) * Hkv
        return {"bytes": float(rows + 2 * sum(lens) * Hkv * d + 8 * blocks + (4 * sum(lens) * Hkv if c["weights"] else 0)), "flops": flops}
    if op == "store":
        n = sum(lens) * Hkv * d
        return {"bytes": float(2 * n * (e + 1)), "flops": 2.0 * n}
    keep = sum(min(n, c["budget"]) for n in lens) * Hkv
    return {"bytes": float(4 * sum(lens) * Hkv + keep * (4 * d + 8)), "flops": 2.0 * keep * d}


# ---- the definitions in 64 bits, one sequence and head at a time


def _e4m3(x):
    """Nearest e4m3 value (ties to even) of 64-bit values up to 448 in magnitude; NaN for what is not finite."""
    _, e = torch.frexp(x)
    step = (((e - 1).clamp(min=-6) - 3 + 1023).long() << 52).view(torch.float64)
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, math.nan)


def _exact_block(value, old, old_scale):
    """Codes of new rows and of older ones [rows, d] (or None) with the scale they share."""
    fine = value[torch.isfinite(value)].abs()
    most = float(fine.max()) if fine.numel() else 0.0
    e = -118
    if most > 0:
        e = max(-118, math.frexp(most)[1] - 9)
        e += 448.0 * 2.0 ** e < most
    scale = 2.0 ** e
    if old is not None and len(old):
        scale = max(scale, old_scale)
        old = _e4m3(old * (old_scale / scale))
    return _e4m3(value / scale), old, scale


def _exact_rows(Q, K, V, limit, scale):
    """O, lse and weights of rows Q [n, d] over K, V [keys, d]; row i sees the first limit[i] keys."""
    O, lse, W = [], [], torch.zeros(K.shape[0], dtype=torch.float64, device=DEV)
    j = torch.arange(K.shape[0], device=DEV)
    for at in range(0, Q.shape[0], 4096):
        S = torch.matmul(Q[at:at + 4096], K.t()) * scale
        S = S.masked_fill(j[None, :] >= limit[at:at + 4096, None], -math.inf)
        l = torch.logsumexp(S, -1)
        P = torch.exp(S - torch.where(l == -math.inf, 0.0, l)[:, None])
        O.append(torch.matmul(P, V))
        lse.append(l)
        W += P.sum(0)
    return torch.cat(O), torch.cat(lse), W


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    op, B, Hkv, G, d = c["op"], c["B"], c["Hkv"], c["G"], c["d"]
    lens = _lens(c)

    def cached(name, table, b, h, n):
        page = c["page"]
        rows = [s[name].view(torch.uint8)[int(p), h].view(F8).double() * float(s[name + "s"][int(p), h])
                for p in table[b, :_pages(n, page)].tolist()]
        rows = [r if name == "K" else r.t() for r in rows]
        return torch.cat(rows)[:n]

    if op in ("prompt", "attend"):
        if op == "attend" and B * Hkv * _pages(c["longest"], c["page"]) > 100000:
            return None
        if op == "prompt" and B * Hkv * G * (c["queries"] or c["longest"]) * c["longest"] * d > 6e11:
            return None
        ql = _q_lens(c)
        O = torch.zeros(s["O"].shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
        W = None if op == "prompt" or s["W"] is None else s["W"].double()
        q0 = k0 = 0
        for b in range(B):
            nq, nk = ql[b], lens[b]
            i = torch.arange(nq, device=DEV)
            limit = i + (nk - nq + 1) if op == "attend" or c["causal"] else torch.full_like(i, nk)
            for h in range(Hkv):
                if op == "prompt":
                    K, V = s["K"][k0:k0 + nk, h].double(), s["V"][k0:k0 + nk, h].double()
                else:
                    K, V = cached("K", s["table"], b, h, nk), cached("V", s["table"], b, h, nk)
                total = torch.zeros(nk, dtype=torch.float64, device=DEV)
                for a in range(h * G, h * G + G):
                    o, l, w = _exact_rows(s["Q"][q0:q0 + nq, a].double(), K, V, limit, s["scale"])
                    O[q0:q0 + nq, a], lse[a, q0:q0 + nq] = o, l
                    total += w
                if W is not None:
                    W[b, h, :nk] = total
            q0, k0 = q0 + nq, k0 + nk
        return (O, lse) if op == "prompt" else (O, lse, W)

    page = c["page"]
    codes = {n: s[n].double() for n in ("K", "V")}
    scales = {n: s[n + "s"].double() for n in ("K", "V")}

    def put(name, p, h, first, rows):
        block = codes[name][p, h] if name == "K" else codes[name][p, h].t()
        block[first:first + rows.shape[0]] = rows

    if op == "store":
        if sum(_pages(n, page) + 1 for n in lens) * Hkv > 30000:
            return None
        k0 = 0
        for b in range(B):
            new, end = lens[b], int(s["lengths"][b])
            start = end - new
            pages = s["table"][b].tolist()
            for j in range(start // page, _pages(end, page)):
                p, lo, hi = pages[j], max(start, j * page), min(end, (j + 1) * page)
                for name, x in (("K", s["Kn"]), ("V", s["Vn"])):
                    rows = x[k0 + lo - start:k0 + hi - start].double()
                    for h in range(Hkv):
                        block = codes[name][p, h] if name == "K" else codes[name][p, h].t()
                        fresh, old, sc = _exact_block(rows[:, h], block[:lo - j * page].clone(), float(scales[name][p, h]))
                        put(name, p, h, 0, old)
                        put(name, p, h, lo - j * page, fresh)
                        scales[name][p, h] = sc
            k0 += new
        return codes["K"], codes["V"], scales["K"], scales["V"]

    if B * Hkv * (_pages(c["longest"], page) + _pages(c["budget"], page)) > 40000:
        return None
    W_to, kept, lengths_to = s["W_to"].double(), s["kept"].clone().fill_(-1), s["lengths_to"].clone()
    for b in range(B):
        n = lens[b]
        keep = min(n, c["budget"])
        recent = min(c["recent"], keep)
        lengths_to[b] = keep
        to = s["to"][b].tolist()
        for h in range(Hkv):
            w = s["W"][b, h, :n].tolist()
            best = sorted(range(n - recent), key=lambda t: (-w[t], t))[:keep - recent]
            at = torch.tensor(sorted(best) + list(range(n - recent, n)), dtype=torch.int64, device=DEV)
            kept[b, h, :keep] = at.int()
            W_to[b, h, :keep] = s["W"][b, h, at].double()
            for name in ("K", "V"):
                rows = cached(name, s["table"], b, h, n)[at]
                for j in range(_pages(keep, page)):
                    code, _, sc = _exact_block(rows[j * page:(j + 1) * page], None, 0.0)
                    put(name, to[j], h, 0, code)
                    scales[name][to[j], h] = sc
    return codes["K"], codes["V"], scales["K"], scales["V"], W_to, kept, lengths_to
