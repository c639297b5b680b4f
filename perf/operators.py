"""The paged cache's operators as cases: block tables and slot maps from request lengths, rows into pages, and attention of the new
tokens of a batch of requests over their pages.

`own` says who computes: the library's entry points (df_page_map, df_paged_append, df_paged_attn) or elementary torch operations in
32 bits.  A case's fields:

    kind      map      block tables extended and slot maps written, from the lengths of the requests
              append   keys and values of the new tokens into the pages that a slot map names
              attn     attention of the new tokens over the pages and over themselves
    heads     "9x1/5 3x0/0" = nine key heads that keep one sink frame and five window frames of T tokens, three that keep
              nothing; "8xfull" = eight that keep every token.  The groups are interleaved.
    group     query heads to a key head
    requests, hist, hist_min, new, new_min, mix
              requests of the batch, cached tokens and new tokens of each: spread over [hist_min, hist] and [new_min, new] by
              `mix`, the first request has the most of both
    block     tokens of a causal block (1: token by token, T: frame by frame), 0: every new token sees all of its request's
    page      tokens of a page
    keys      whether the new tokens have keys of their own (False: they only look back)
    lse       whether the log-sum-exp is wanted
"""
import random

import torch

own = False

_DEVICE = "cuda"
_FULL = 1 << 30                                              # window of a head that keeps every token


def listed():
    def case(name, kind, heads, requests, hist, new, group=1, T=1, d=128, hist_min=None, new_min=None, mix=0, block=1, page=64,
             dtype="bfloat16", keys=True, lse=False):
        return dict(name=name, kind=kind, heads=heads, requests=requests, hist=hist, new=new, group=group, T=T, d=d,
                    hist_min=hist if hist_min is None else hist_min, new_min=new if new_min is None else new_min, mix=mix, block=block,
                    page=page, dtype=dtype, keys=keys, lse=lse)

    return [
        # one step of a token server: 64 requests get a token each, small pages, now and then a new page
        case("map_tokens", "map", "8xfull", 64, 8192, 1, hist_min=1, mix=1, page=16),
        # six videos finish an 832x480 chunk: heads of four types, tens of thousands of slots
        case("map_chunks_480p", "map", "3x1/5 3x1/0 3x0/5 3x0/1", 6, 14040, 4680, T=1560, hist_min=0, mix=2),
        # the rows of 64 single tokens: latency
        case("append_tokens", "append", "8xfull", 64, 2048, 1, hist_min=1, mix=3, page=16),
        # two finished 1280x720 chunks, a quarter of the heads keeps nothing: a large copy
        case("append_chunks_720p", "append", "9x1/11 3x0/0", 2, 43200, 10800, T=3600, mix=4),
        # the smallest attention: one request, four narrow heads, one token, three frames of 64 tokens behind it
        case("token_tiny_d64", "attn", "4xfull", 1, 192, 1, d=64, mix=5),
        # a serving batch, one token each, grouped heads, ragged lengths up to 8192, small pages
        case("tokens_batch", "attn", "8xfull", 64, 8192, 1, group=4, hist_min=1, mix=6, page=16),
        # one token of one request with a long cache
        case("token_long", "attn", "8xfull", 1, 131072, 1, group=4, mix=7),
        # five drafted tokens of 16 requests to be verified, fp16, with the log-sum-exp
        case("draft_fp16", "attn", "8xfull", 16, 16384, 5, group=4, hist_min=100, mix=8, page=32, dtype="float16", lse=True),
        # prompts taken in ragged pieces, causal token by token, one request with a single token among them
        case("prompt_pieces", "attn", "8xfull", 5, 6000, 2048, group=4, hist_min=0, new_min=1, mix=9, page=16),
        # four 390-token-a-frame previews at different places, causal frame by frame, narrow heads of all types, fp16
        case("preview_frames_d64", "attn", "3x1/5 2x1/0 3x0/5 2x0/0 2x0/1", 4, 3900, 1170, T=390, d=64, hist_min=0, mix=10, block=390,
             dtype="float16", lse=True),
        # two 832x480 chunks whose windows have wrapped, a quarter of the heads keeps no history
        case("chunks_480p", "attn", "9x1/5 3x0/0", 2, 14041, 4680, T=1560, mix=11, block=0),
        # one 1280x720 chunk with twelve cached frames: the largest
        case("chunk_720p", "attn", "9x1/11 3x0/0", 1, 43200, 10800, T=3600, mix=12, block=0),
    ]


def _contexts(case):
    """(sink, window) in tokens of every key head, the groups interleaved."""
    groups = []
    for part in case["heads"].split():
        n, ctx = part.split("x")
        s, w = (0, _FULL) if ctx == "full" else (int(x) * case["T"] for x in ctx.split("/"))
        groups.append((int(n), s, w))
    spread = [((i + 0.5) / n, g, s, w) for g, (n, s, w) in enumerate(groups) for i in range(n)]
    return [(s, w) for _, _, s, w in sorted(spread)]


def _lengths(case):
    """Cached and new tokens of every request."""
    rng = random.Random(case["mix"])
    hist = [rng.randint(case["hist_min"], case["hist"]) for _ in range(case["requests"])]
    new = [rng.randint(case["new_min"], case["new"]) for _ in range(case["requests"])]
    return [case["hist"]] + hist[1:], [case["new"]] + new[1:]


def _pairs(case):
    """(visible keys over all queries, keys some query sees) of one request and key head, summed over both."""
    hist, new = _lengths(case)
    pairs = keys = 0
    for L, n in zip(hist, new):
        block = case["block"] or n
        for s, w in _contexts(case):
            held = min(L, s) + min(max(L - s, 0), w)
            keys += held + (n if case["keys"] else 0)
            for first in range(0, n, block):
                last = min(first + block, n)
                back = min(L, s) + max(0, L - max(s, L + first - w))
                ahead = last - max(0, first - w) + min(max(0, first - w), max(0, s - L)) if case["keys"] else 0
                pairs += (last - first) * (back + ahead)
    return pairs, keys


def work(case):
    ctx, (hist, new) = _contexts(case), _lengths(case)
    total, row = sum(new), 2 * case["d"]
    if case["kind"] == "map":
        return {"bytes": 8 * total * len(ctx) + 12 * len(hist), "flops": 10 * total * len(ctx)}
    if case["kind"] == "append":
        kept = sum(min(n, max(0, s - L) + min(w, n - min(n, max(0, s - L)))) for L, n in zip(hist, new) for s, w in ctx)
        return {"bytes": 4 * row * kept + 8 * total * len(ctx), "flops": 0}
    pairs, keys = _pairs(case)
    heads = len(ctx) * case["group"]
    return {"bytes": row * (2 * total * heads + 2 * keys) + 4 * total * heads * case["lse"], "flops": 4 * case["d"] * case["group"] * pairs}


def draw(rng):
    largest = work(listed()[-1])

    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    while True:
        kind = rng.choice(["map", "append", "attn", "attn", "attn", "attn"])
        use = rng.choice(["token", "draft", "pieces", "video", "video"])
        T, block, keys, group, requests = 1, 1, True, rng.choice([1, 2, 4, 5, 8]), spread(1, 96)
        if use == "video":
            T, group, requests = spread(33, 3600), rng.choice([1, 1, 1, 2]), spread(1, 6)
            frames, n_heads = spread(1, 24), rng.choice([2, 5, 8, 12, 12, 24])
            kinds = ["1/%d" % frames, "1/0", "0/%d" % frames, "0/0", "0/1"]
            picked = [rng.choice(kinds) for _ in range(n_heads)]
            heads = " ".join("%dx%s" % (picked.count(k), k) for k in kinds if k in picked)
            new, hist = rng.choice([1, 2, 3]) * T, int(rng.uniform(0, frames + 4) * T)
            block, keys = rng.choice([0, T]), rng.random() < 0.9
            new_min = rng.choice([new, T])
        else:
            heads = "%dxfull" % rng.choice([1, 2, 4, 7, 8, 12])
            new = {"token": 1, "draft": spread(2, 16), "pieces": spread(17, 4096)}[use]
            new_min, hist = rng.choice([1, new]), spread(1, 200000 // requests)
            if use == "pieces":
                requests, hist = min(requests, 8), min(hist, 32768)
        case = dict(kind=kind, heads=heads, requests=requests, hist=hist, new=new, group=group, T=T, d=rng.choice([64, 128, 128]),
                    hist_min=rng.choice([0, hist // 2, hist]), new_min=new_min, mix=rng.randrange(1 << 20), block=block,
                    page=rng.choice([16, 32, 64, 64, 128]), dtype=rng.choice(["bfloat16", "bfloat16", "float16"]),
                    keys=keys or kind != "attn", lse=kind == "attn" and rng.random() < 0.4)
        w = work(case)
        scores = 4 * requests * len(_contexts(case)) * group * new * (hist + 2 * new)
        if w["flops"] <= largest["flops"] and w["bytes"] <= 1.5e9 and scores <= 40e9:
            return case


def prepare(case, seed):
    """A pool of pages in which the requests' pages lie anywhere, their block tables and lengths, and the new tokens."""
    ctx, (hist, new) = _contexts(case), _lengths(case)
    Hkv, P, d, dtype, B = len(ctx), case["page"], case["d"], getattr(torch, case["dtype"]), case["requests"]
    total = sum(new)
    g = torch.Generator(device=_DEVICE).manual_seed(seed)

    def gauss(*shape):
        return torch.randn(*shape, generator=g, device=_DEVICE, dtype=dtype)

    held = torch.tensor([[-(-min(L, s + w) // P) for s, w in ctx] for L in hist])
    after = torch.tensor([[-(-min(L + n, s + w) // P) for s, w in ctx] for L, n in zip(hist, new)])
    max_pages, n_held = max(1, int(after.max())), int(held.sum())
    n_pages = n_held + int((after - held).sum()) + 7
    order = torch.randperm(n_pages, generator=g, device=_DEVICE).to(torch.int32)
    table = torch.full((B, Hkv, max_pages), -1, dtype=torch.int32, device=_DEVICE)
    table[(torch.arange(max_pages) < held[:, :, None]).to(_DEVICE)] = order[:n_held]
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=_DEVICE)
    free[: n_pages - n_held] = order[n_held:]
    cum = [0]
    for n in new:
        cum.append(cum[-1] + n)

    def ints(x, t=torch.int32):
        return torch.tensor(x, dtype=t, device=_DEVICE)

    st = dict(kind=case["kind"], P=P, d=d, dtype=dtype, total=total, block=case["block"] or case["new"], new=case["new"], keys=case["keys"],
              group=case["group"], scale=d ** -0.5, table=table, length=ints(hist), cu_new=ints(cum), sink=ints([s for s, _ in ctx]),
              window=ints([w for _, w in ctx]), free=free, n_free=ints([n_pages - n_held]))
    if case["kind"] == "map":
        # pages are not touched by a map; a program has the pool all the same
        st.update(k_pages=torch.zeros(n_pages, P, d, dtype=dtype, device=_DEVICE), len_out=ints([0] * B), n_free_out=ints([0]),
                  status=ints([0]), slots=torch.zeros(total, Hkv, dtype=torch.int64, device=_DEVICE))
        st["v_pages"] = st["k_pages"]
        return st
    st.update(k_pages=gauss(n_pages, P, d), v_pages=gauss(n_pages, P, d))
    st.update(k_new=gauss(total, Hkv, d), v_new=gauss(total, Hkv, d))
    if case["kind"] == "append":
        st["slots"] = _slots(st)[0]
        return st
    Hq = Hkv * case["group"]
    mean = 0.4 * torch.randn(Hq, d, generator=g, device=_DEVICE)
    st["q"] = (torch.randn(total, Hq, d, generator=g, device=_DEVICE) + mean).to(dtype)
    st["out"] = torch.empty_like(st["q"])
    st["lse"] = torch.empty(Hq, total, dtype=torch.float32, device=_DEVICE) if case["lse"] else None
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------------

def _owners(st):
    """Request and place in its request of every new token."""
    t = torch.arange(st["total"], device=_DEVICE)
    b = torch.searchsorted(st["cu_new"].long(), t, right=True) - 1
    return b, t - st["cu_new"].long()[b]


def _held(st, length):
    """Filled slots [requests, heads] after `length` tokens."""
    return torch.minimum(length[:, None].long(), st["sink"].long() + st["window"].long())


def _slots(st):
    """Slot map, table, lengths, free pages left and status."""
    P, table, free = st["P"], st["table"].long(), st["free"].long()
    new = (st["cu_new"][1:] - st["cu_new"][:-1]).long()
    length, sink, window = st["length"].long(), st["sink"].long(), st["window"].long()
    before = (_held(st, length) + P - 1) // P
    after = (_held(st, length + new) + P - 1) // P
    need = after - before
    begin = need.flatten().cumsum(0).reshape(need.shape) - need
    n_free = st["n_free"].long()
    good = (need.sum() <= n_free) & (after <= table.shape[2]).all()
    page = torch.arange(table.shape[2], device=_DEVICE)
    place = n_free - 1 - begin[:, :, None] - (page - before[:, :, None])
    added = good & (page >= before[:, :, None]) & (page < after[:, :, None])
    table = torch.where(added, free[place.clamp(0, free.numel() - 1)], table)
    b, i = _owners(st)
    j = (length[b] + i)[:, None]
    slot = torch.where(j < sink, j, sink + (j - sink) % window.clamp(min=1))
    kept = good & ((j < sink) | (j >= (length + new)[b][:, None] - window) & (window > 0))
    entry = table[b[:, None], torch.arange(sink.numel(), device=_DEVICE), (slot // P).clamp(max=table.shape[2] - 1)]
    slots = torch.where(kept, entry * P + slot % P, -1)
    left = n_free - torch.where(good, need.sum(), 0)
    return slots, table.int(), torch.where(good, length + new, length).int(), left.int(), torch.where(good, 0, 6).int().reshape(1)


def _append(st):
    kept = st["slots"] >= 0
    at = st["slots"][kept]
    st["k_pages"].view(-1, st["d"])[at] = st["k_new"][kept]
    st["v_pages"].view(-1, st["d"])[at] = st["v_new"][kept]
    return [st["k_pages"], st["v_pages"]]


def _attention(st):
    table, d, group = st["table"].long(), st["d"], st["group"]
    B, Hkv, M = table.shape
    b, i = _owners(st)
    n_max, block = st["new"], st["block"]
    new = (st["cu_new"][1:] - st["cu_new"][:-1]).long()[:, None, None, None]
    L, sink, window = st["length"].long()[:, None, None, None], st["sink"].long()[None, :, None, None], st["window"].long()[None, :, None, None]

    def pages(pool):                                         # [B, Hkv, slots, d]
        return pool[table.clamp(min=0)].reshape(B, Hkv, -1, d)

    rows = (st["cu_new"][:-1].long()[:, None] + torch.arange(n_max, device=_DEVICE)).clamp(max=st["total"] - 1)
    q = st["q"][rows].float().reshape(B, n_max, Hkv, group, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, group * n_max, d)
    # the position that a slot holds, and who sees it
    r = torch.arange(M * st["P"], device=_DEVICE)
    turn = (L - sink).clamp(min=0)
    at = turn % window.clamp(min=1)
    k = r - sink
    ring = torch.where(k < at, L - at + k, L - at - window + k)
    position = torch.where((r < sink) | (turn <= window), r, ring)
    held = r < torch.minimum(L, sink + window)
    x = torch.arange(n_max, device=_DEVICE)[:, None]
    first = x // block * block
    sees = held & ((position < sink) | (position >= L + first - window))
    k_all, v_all = pages(st["k_pages"]), pages(st["v_pages"])
    v_all = v_all.masked_fill(~held.reshape(B, Hkv, -1, 1), 0.0)
    if st["keys"]:
        t = torch.arange(n_max, device=_DEVICE)
        ahead = (t < torch.minimum(first + block, new)) & ((t >= first - window) | (L + t < sink))
        sees = torch.cat([sees, ahead], 3)
        k_all = torch.cat([k_all, st["k_new"][rows].transpose(1, 2)], 2)
        v_all = torch.cat([v_all, st["v_new"][rows].transpose(1, 2)], 2)
    scores = torch.matmul(q, k_all.float().transpose(2, 3)).mul_(st["scale"]).reshape(B, Hkv, group, n_max, -1)
    scores.masked_fill_(~sees[:, :, None], float("-inf"))
    most = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = scores.sub_(most).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.reshape(B, Hkv, group * n_max, -1), v_all.float()).reshape(B, Hkv, group, n_max, d)
    out = torch.where(total > 0, out / total, 0.0).to(st["dtype"])
    out = out[b, :, :, i].reshape(st["total"], Hkv * group, d)
    if st["lse"] is None:
        return [out]
    lse = (most + total.log())[..., 0]
    return [out, lse[b, :, :, i].reshape(st["total"], Hkv * group).t().contiguous()]


# ---- the library's calls ------------------------------------------------------------------------------------------------------

def _handle(st):
    """The cache's handle and the workspace, made by the first call as by a program's set-up."""
    from paper_2601_20499_amd import binding as df
    if "cache" not in st:
        st["cache"] = df.PagedCache(st["k_pages"], st["v_pages"], st["table"], st["length"], st["sink"], st["window"], st["free"], st["n_free"])
        if st["kind"] == "attn":
            n = df.df_paged_workspace_bytes(st["q"].shape[1], st["cache"].Hkv, st["d"], st["new"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device=_DEVICE)
    return df, st["cache"]


def run(st):
    if not own:
        if st["kind"] == "map":
            return list(_slots(st))
        return _append(st) if st["kind"] == "append" else _attention(st)
    df, cache = _handle(st)
    if st["kind"] == "map":
        df.df_page_map(cache, st["cu_new"], st["slots"], st["status"], len_out=st["len_out"], n_free_out=st["n_free_out"])
        return [st["slots"], st["table"], st["len_out"], st["n_free_out"], st["status"]]
    if st["kind"] == "append":
        df.df_paged_append(cache, st["k_new"], st["v_new"], st["slots"])
        return [st["k_pages"], st["v_pages"]]
    df.df_paged_attn(st["q"], st["k_new"] if st["keys"] else None, st["v_new"] if st["keys"] else None, cache, st["cu_new"], st["out"],
                     st["scale"], block=st["block"], max_new=st["new"], lse_out=st["lse"], workspace=st["ws"])
    return [st["out"]] if st["lse"] is None else [st["out"], st["lse"]]


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------------------

def exact(case, seed):
    """Request by request and head by head: the pools after an append; outputs of attention, each from the list of the positions
    that a head holds.  A map gives whole numbers."""
    if case["kind"] == "map":
        return None
    st = prepare(case, seed)
    ctx, (hist, new) = _contexts(case), _lengths(case)
    if case["kind"] == "append":
        k, v, start = st["k_pages"].double(), st["v_pages"].double(), 0
        for L, n in zip(hist, new):
            for h, (s, w) in enumerate(ctx):
                t = torch.cat([torch.arange(0, min(n, max(0, s - L))), torch.arange(min(n, max(0, s - L, n - w)), n)]).to(_DEVICE)
                at = st["slots"][start + t, h]
                k.view(-1, case["d"])[at], v.view(-1, case["d"])[at] = st["k_new"][start + t, h].double(), st["v_new"][start + t, h].double()
            start += n
        return [k, v]
    d, P, group, dev = case["d"], case["page"], case["group"], _DEVICE
    out = torch.empty(st["total"], len(ctx) * group, d, dtype=torch.float64, device=dev)
    lse = torch.empty(len(ctx) * group, st["total"], dtype=torch.float64, device=dev)
    start = 0
    for req, (L, n) in enumerate(zip(hist, new)):
        block = case["block"] or n
        for h, (s, w) in enumerate(ctx):
            at = torch.cat([torch.arange(0, min(L, s), device=dev), torch.arange(max(min(L, s), L - w), L, device=dev)])
            slot = torch.where(at < s, at, s + (at - s) % max(w, 1))
            row = st["table"][req, h, slot // P].long() * P + slot % P
            keys, vals = st["k_pages"].view(-1, d)[row].double(), st["v_pages"].view(-1, d)[row].double()
            if case["keys"]:
                keys = torch.cat([keys, st["k_new"][start:start + n, h].double()])
                vals = torch.cat([vals, st["v_new"][start:start + n, h].double()])
                at = torch.cat([at, torch.arange(L, L + n, device=dev)])
            heads = slice(h * group, (h + 1) * group)
            step = max(1, 50_000_000 // (group * max(1, len(at))))
            for lo in range(0, n, step):
                hi = min(n, lo + step)
                i = torch.arange(lo, hi, device=dev)[:, None]
                first = i // block * block
                sees = (at < L + (first + block).clamp(max=n)) & ((at < s) | (at >= L + first - w))
                q = st["q"][start + lo:start + hi, heads].double().transpose(0, 1)
                logits = (q @ keys.t() * st["scale"]).masked_fill(~sees, float("-inf"))
                total = torch.logsumexp(logits, 2, keepdim=True)
                p = (logits - total).exp().masked_fill(~sees, 0.0)
                out[start + lo:start + hi, heads] = (p @ vals).transpose(0, 1)
                lse[heads, start + lo:start + hi] = total[..., 0]
        start += n
    return [out, lse] if case["lse"] else [out]
