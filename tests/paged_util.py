"""A batch of requests over a paged cache, the plain way: the oracle of the paged operators' tests.

Pages and slots are kept in python lists, token by token; attention is written out in 64 bits, row by row of what a query sees.  Nothing
here is shared with the library."""
import numpy as np
import torch

FULL = 1 << 30                                   # window of a head that keeps every token


class Model:
    """Tokens by position, and for every (request, head) its pages in order."""

    def __init__(self, B, caps, n_pages, page, max_pages, free=None):
        self.B, self.H, self.page, self.max_pages, self.n_pages = B, len(caps[0]), page, max_pages, n_pages
        self.caps = caps                         # [request][head] = (sink, window)
        self.len = [0] * B
        self.pages = [[[] for _ in range(self.H)] for _ in range(B)]
        self.free = list(range(n_pages)) if free is None else list(free)
        self.kept = {}                           # (request, head) -> {slot: (k row, v row)}, filled by put()

    @staticmethod
    def slot(j, s, w):
        return j if j < s else s + (j - s) % w if w else None

    def map(self, new, release=None):
        """Slots [token][head] of the new tokens (-1: not kept), or None if the step cannot be done (then nothing changes)."""
        release = release or [0] * self.B
        free, pages, length = list(self.free), [[list(x) for x in r] for r in self.pages], list(self.len)
        for b in range(self.B):
            if release[b]:
                for h in range(self.H):
                    free += pages[b][h]
                    pages[b][h] = []
                length[b] = 0
        slots = []
        for b in range(self.B):
            after = length[b] + new[b]
            rows = [[-1] * self.H for _ in range(new[b])]
            for h, (s, w) in enumerate(self.caps[b]):
                need = -(-min(after, s + w) // self.page)
                if need > self.max_pages:
                    return None
                while len(pages[b][h]) < need:
                    if not free:
                        return None
                    pages[b][h].append(free.pop())
                for i in range(new[b]):
                    j = length[b] + i
                    if j < s or (w and j >= after - w):
                        x = self.slot(j, s, w)
                        rows[i][h] = pages[b][h][x // self.page] * self.page + x % self.page
            slots += rows
            length[b] = after
        self.free, self.pages, self.len = free, pages, length
        return slots


def held_positions(L, s, w):
    """Positions that a head holds of L tokens, ascending."""
    return list(range(min(L, s))) + list(range(max(min(L, s), L - w), L))


def attend(q, k, v, scale):
    """One query row against the keys it sees, in 64 bits: output, weights' sum of |v| (for the error bound), log-sum-exp."""
    if k.shape[0] == 0:
        return np.zeros(q.shape[-1]), np.zeros(q.shape[-1]), -np.inf
    s = scale * (k @ q)
    m = s.max()
    p = np.exp(s - m)
    return p @ v / p.sum(), p @ np.abs(v) / p.sum(), m + np.log(p.sum())


class Batch:
    """Device tensors of one attention call, made from positions: histories that lie in random pages, stale rows of which hold
    `stale`."""

    def __init__(self, seed, lens, new, caps, G=1, d=128, dtype=torch.bfloat16, page=16, keys=True, stale=float("nan"), spare=3,
                 device="cuda:0", table_extra=1, q_mean=0.3):
        g = torch.Generator().manual_seed(seed)
        B, H = len(lens), len(caps[0]) if isinstance(caps[0][0], tuple) else len(caps)
        self.per_request = isinstance(caps[0][0], tuple)
        self.caps = caps if self.per_request else [list(caps)] * B
        self.B, self.H, self.G, self.d, self.dtype, self.page, self.keys = B, H, G, d, dtype, page, keys
        self.lens, self.new, self.scale = list(lens), list(new), d ** -0.5
        total = sum(new)
        rnd = lambda *s: torch.randn(*s, generator=g).to(dtype)
        self.hist = [[(rnd(L, d), rnd(L, d)) for _ in range(H)] for L in lens]      # whole histories; only what is held lies in pages
        self.k_new, self.v_new = rnd(total, H, d), rnd(total, H, d)
        self.q = (torch.randn(total, H * G, d, generator=g) + q_mean).to(dtype)
        pages = [[-(-min(L, s + w) // page) for s, w in self.caps[b]] for b, L in enumerate(lens)]
        n_pages = sum(map(sum, pages)) + spare
        self.max_pages = max(1, max(map(max, pages))) + table_extra
        order = torch.randperm(n_pages, generator=g).tolist()
        k = torch.full((n_pages, page, d), stale, dtype=dtype)
        v = torch.full((n_pages, page, d), stale, dtype=dtype)
        table = torch.full((B, H, self.max_pages), -(1 << 30), dtype=torch.int32)
        for b, L in enumerate(lens):
            for h, (s, w) in enumerate(self.caps[b]):
                own = [order.pop() for _ in range(pages[b][h])]
                table[b, h, :len(own)] = torch.tensor(own, dtype=torch.int32)
                at = held_positions(L, s, w)
                if at:
                    slot = torch.tensor([Model.slot(j, s, w) for j in at])
                    row = torch.tensor(own)[slot // page] * page + slot % page
                    k.view(-1, d)[row] = self.hist[b][h][0][at]
                    v.view(-1, d)[row] = self.hist[b][h][1][at]
        put = lambda t: t.to(device)
        self.dev = device
        self.k_pages, self.v_pages, self.table = put(k), put(v), put(table)
        self.length = torch.tensor(lens, dtype=torch.int32, device=device)
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=device)
        cap = torch.tensor(self.caps if self.per_request else self.caps[0], dtype=torch.int32)
        self.sink, self.win = put(cap[..., 0].contiguous()), put(cap[..., 1].contiguous())
        free = torch.full((n_pages,), -1, dtype=torch.int32)
        free[:len(order)] = torch.tensor(order, dtype=torch.int32)
        self.free, self.n_free = put(free), torch.tensor([len(order)], dtype=torch.int32, device=device)

    def cache(self, df):
        return df.PagedCache(self.k_pages, self.v_pages, self.table, self.length, self.sink, self.win, self.free, self.n_free)

    def run(self, df, block, lse=True, extra_rows=0, max_new=None, fill=7.0, cache=None, stream=None, ws=None):
        """Output and log-sum-exp of the call; `extra_rows` rows of no request follow the batch, filled with `fill`."""
        put = lambda t: torch.cat([t, torch.full((extra_rows, *t.shape[1:]), float("nan"), dtype=t.dtype)]).to(self.dev)
        q = put(self.q)
        out = torch.full_like(q, fill)
        ls = torch.full((q.shape[1], q.shape[0]), fill, dtype=torch.float32, device=self.dev) if lse else None
        most = max(max(self.new), 1) if max_new is None else max_new
        if ws is None:
            ws = torch.full((df.df_paged_workspace_bytes(self.H * self.G, self.H, self.d, most),), 0x5A, dtype=torch.uint8, device=self.dev)
        kc, vc = (put(self.k_new), put(self.v_new)) if self.keys else (None, None)
        df.df_paged_attn(q, kc, vc, cache or self.cache(df), self.cu, out, self.scale, block=block, max_new=most, lse_out=ls, workspace=ws,
                         stream=stream)
        return out, ls

    def sees(self, b, h, i, block):
        """History positions and new tokens that query i of request b sees in key head h."""
        s, w = self.caps[b][h]
        L, n = self.lens[b], self.new[b]
        first = i // block * block
        back = [j for j in held_positions(L, s, w) if j < s or j >= L + first - w]
        ahead = [t for t in range(min(first + block, n)) if t >= first - w or L + t < s] if self.keys else []
        return back, ahead

    def reference(self, block, rows=None):
        """(out, sum of weights |v|, lse, keys, sum |q k|) in 64 bits, of the token rows `rows` (default all)."""
        total, Hq = self.q.shape[0], self.H * self.G
        out, mag = np.zeros((total, Hq, self.d)), np.zeros((total, Hq, self.d))
        lse, n_keys, reach = np.full((Hq, total), -np.inf), np.zeros((Hq, total)), np.zeros((Hq, total))
        q = self.q.double().numpy()
        start = 0
        for b, n in enumerate(self.new):
            seen_by = {}
            for i in range(n):
                if rows is not None and start + i not in rows:
                    continue
                for h in range(self.H):
                    key = (h, i // block)
                    if key not in seen_by:
                        back, ahead = self.sees(b, h, i, block)
                        at = [start + t for t in ahead]
                        seen_by[key] = [np.concatenate([self.hist[b][h][x][back].double().numpy(), y[at, h].double().numpy()])
                                        for x, y in ((0, self.k_new), (1, self.v_new))]
                    k, v = seen_by[key]
                    for hq in range(h * self.G, (h + 1) * self.G):
                        out[start + i, hq], mag[start + i, hq], lse[hq, start + i] = attend(q[start + i, hq], k, v, self.scale)
                        n_keys[hq, start + i] = len(k)
                        reach[hq, start + i] = self.scale * (np.abs(k) @ np.abs(q[start + i, hq])).max(initial=0.0)
            start += n
        return out, mag, lse, n_keys, reach


def bounds(ref, dtype, d):
    """Largest error of output and log-sum-exp, element by element.

    A score is a sum of d products in 32 bits: off by at most d 2^-24 of the sum of their sizes (`reach`), in natural units; a weight by
    twice that (it and the reference's), by the exponential's last bit and by the rounding of score * c (|score| <= reach): together e.
    The weight then is rounded to the type (half a step, eps / 2), an output is a sum of weighted values over the sum of weights
    (off by e + eps / 2 of sum(weight |v|)) in up to `keys` 32-bit additions (taken 8 at a time by the matrix core: keys / 8 roundings
    of 2^-24, and 2^-20 for pieces put together), rounded once (eps / 2 of itself).  fp16 weights below 2^-14 of the
    reference and results below 2^-14 are off by up to half the smallest step, 2^-25.  The log-sum-exp has e, the additions and
    a few steps of itself."""
    out, mag, lse, keys, reach = ref
    half = torch.finfo(dtype).eps / 2
    e = (2 * d + 16) * 2.0 ** -24 * (reach + 1) + keys / 8 * 2.0 ** -24 + 2.0 ** -20
    e_row = e.T[:, :, None]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    big = mag.max(-1, keepdims=True)
    tol = (e_row + half) * mag * (1 + half) + half * np.abs(out) + tiny * (1 + keys.T[:, :, None] * big) + 1e-30
    tol_lse = e + 8 * 2.0 ** -24 * np.where(np.isfinite(lse), np.abs(lse), 0) + 2.0 ** -22
    return tol, tol_lse


def check(out, lse, ref, dtype, d, what="", rows=None):
    tol, tol_lse = bounds(ref, dtype, d)
    got = out.double().cpu().numpy()[: ref[0].shape[0]]
    sel = slice(None) if rows is None else np.array(sorted(rows))
    err = np.abs(got - ref[0])[sel]
    worst = (err / tol[sel]).max() if err.size else 0.0
    msg = f"{what}: max|err|={err.max() if err.size else 0:.2e}, {worst:.2f} of the bound"
    if lse is not None:
        l = lse.double().cpu().numpy()[:, : ref[2].shape[1]][:, sel]
        want = ref[2][:, sel]
        assert np.array_equal(np.isneginf(l), np.isneginf(want)), what
        fin = np.isfinite(want)
        el = np.abs(l[fin] - want[fin]) / tol_lse[:, sel][fin]
        msg += f"; lse {el.max() if el.size else 0:.2f}"
        assert not el.size or (np.isfinite(el).all() and el.max() <= 1), msg
    print(msg, flush=True)
    assert np.isfinite(got[sel]).all() and worst <= 1, msg
