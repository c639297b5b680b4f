"""The paged operators where they can go wrong: values that are not numbers, pages that are none, climbing scores, other layouts, long and far
caches, other streams, captured steps, and whole loops of them."""
import numpy as np
import pytest
import torch

from tests import paged_util as pu
from tests.paged_util import FULL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16 = torch.bfloat16, torch.float16
ALL = 1 << 30


@pytest.fixture(scope="module")
def df():
    from paper_2601_20499_amd import binding
    return binding


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def run(df, b, block, **kw):
    out = b.run(df, block, **kw)
    torch.cuda.synchronize()
    return out


def in_pages(b, r, h, j):
    """(page, row) of the kept position j."""
    slot = pu.Model.slot(j, *b.caps[r][h])
    return int(b.table[r, h, slot // b.page]), slot % b.page


def repack(b):
    """Writes the histories of the batch to its pages again."""
    for r, L in enumerate(b.lens):
        for h, (s, w) in enumerate(b.caps[r]):
            for j in pu.held_positions(L, s, w):
                page, row = in_pages(b, r, h, j)
                b.k_pages[page, row], b.v_pages[page, row] = b.hist[r][h][0][j].to(DEV), b.hist[r][h][1][j].to(DEV)


# (new tokens, query heads to a key head, block): up to 32 rows, and more
KINDS = {"few": (6, 4, 2), "many": (150, 1, 40)}


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, FP16)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_seen_has_no_influence(df, kind, d, dtype, odd):
    """A value that is no number, in a new token and in the cache, is in the results of those rows that see it, and in their column only."""
    n, G, block = KINDS[kind]
    b = pu.Batch(5, [100], [n], [(0, FULL), (8, 30)], G, d, dtype)
    base, lse = run(df, b, block)
    t = n - 2 * block + 1
    b.v_new[t, :, 5] = odd
    spoiled = []
    for h, j in ((0, 3), (1, 72)):                     # seen by all blocks, and not by the last
        page, row = in_pages(b, 0, h, j)
        b.v_pages[page, row, 9] = odd
        spoiled.append(j)
    got, lse2 = run(df, b, block)
    assert torch.equal(lse, lse2)
    kinds = set()
    for h in range(2):
        for i in range(n):
            back, ahead = b.sees(0, h, i, block)
            for hq in range(h * G, h * G + G):
                want = base[i, hq].clone()
                if t in ahead:
                    want[5] = odd
                if spoiled[h] in back:
                    want[9] = odd
                kinds.add((h, t in ahead, spoiled[h] in back))
                assert torch.equal(got[i, hq].nan_to_num(1e4, 3e4, -3e4), want.nan_to_num(1e4, 3e4, -3e4)), (h, i, hq)
    assert {(0, False, True), (0, True, True)} <= kinds and len({x[2] for x in kinds if x[0] == 1}) == 2


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, FP16)])
@pytest.mark.parametrize("kind", KINDS)
def test_keys_that_are_no_numbers(df, kind, d, dtype):
    n, G, block = KINDS[kind]
    b = pu.Batch(6, [70], [n], [(0, FULL), (8, 30)], G, d, dtype)
    ref = b.reference(block)
    t = n - 2 * block + 1
    b.k_new[t] = float("nan")
    out, lse = run(df, b, block)
    for h in range(2):
        heads = slice(h * G, h * G + G)
        blind = [i for i in range(n) if t not in b.sees(0, h, i, block)[1]]
        rest = [i for i in range(n) if i not in blind]
        part = tuple(x[:, heads] if x.shape[0] == n else x[heads] for x in ref)
        pu.check(out[:, heads], lse[heads], part, dtype, d, "%s head %d" % (kind, h), rows=blind)
        assert rest and out[rest, heads].isnan().all() and lse[heads][:, rest].isnan().all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("keys", [True, False])
def test_scores_of_minus_infinity(df, kind, keys):
    """A row all of whose keys score minus infinity is 0, and one of whose keys does not is not changed by the others."""
    n, G, block = KINDS[kind]
    b = pu.Batch(7, [90, 33, 0], [n, n, n], [(0, FULL)] * 2, G, 64, BF16, keys=keys)
    b.q[..., 0] = b.q[..., 0].abs() + 0.1
    for r in range(3):
        for h in range(2):
            b.hist[r][h][0][: 80 if r == 0 else 33, 0] = float("-inf")       # request 0 keeps ten ordinary keys
    if keys:
        b.k_new[n:, :, 0] = float("-inf")
    repack(b)
    out, lse = run(df, b, block)
    for k in [b.hist[r][h][0] for r in range(3) for h in range(2)] + [b.k_new]:
        k[k.isneginf()] = -60000.0                     # exp of it is 0 in 64 bits too
    rows = list(range(n))
    ref = b.reference(block, rows)
    # the sizes of the scores that are not minus infinity bound the errors
    real = np.abs(np.concatenate([b.hist[0][0][0][80:].double().numpy(), b.hist[0][1][0][80:].double().numpy(), b.k_new[:n].double().numpy().reshape(-1, 64)]))
    reach = b.scale * np.einsum("ihd,kd->hik", np.abs(b.q[:n].double().numpy()), real).max(-1)
    ref[4][:, :n] = reach
    pu.check(out, lse, ref, BF16, 64, kind, rows=rows)
    assert (out[n:] == 0).all() and lse[:, n:].isneginf().all()


@pytest.mark.parametrize("bad", [-1, -(1 << 31), "n_pages", (1 << 31) - 1])
@pytest.mark.parametrize("kind", KINDS)
def test_a_page_that_is_none(df, kind, bad):
    n, G, _ = KINDS[kind]
    b = pu.Batch(8, [200, 50], [n, n], [(0, FULL)] * 3, G, 128, BF16)
    base, lse = run(df, b, ALL)
    b.table[0, 1, 7] = b.k_pages.shape[0] if bad == "n_pages" else bad
    out, lse2 = run(df, b, ALL)
    spoiled = torch.zeros(out.shape[:2], dtype=torch.bool, device=DEV)
    spoiled[:n, G:2 * G] = True
    assert out[spoiled].isnan().all() and lse2.T[spoiled].isnan().all()
    assert torch.equal(out[~spoiled], base[~spoiled]) and torch.equal(lse2.T[~spoiled], lse.T[~spoiled])


@pytest.mark.parametrize("kind", KINDS)
def test_lengths_out_of_range(df, kind):
    n, G, block = KINDS[kind]
    b = pu.Batch(9, [60, 50, 0], [n, n, n], [(0, FULL), (3, 20)], G, 64, BF16)
    base, lse = run(df, b, block)
    b.length[0] = (1 << 31) - 1                        # more than the table's pages
    b.length[2] = -5                                   # none
    out, lse2 = run(df, b, block)
    assert torch.equal(out[n:], base[n:]) and torch.equal(lse2[:, n:], lse[:, n:])
    assert out[:n, :G].isnan().all() and lse2[:G, :n].isnan().all()


PROFILES = {"stairs": lambda j: 12.0 * (j // 32), "second halves": lambda j: 12.0 * ((j + 32) // 64), "one peak": lambda j: np.where(j == 201, 40.0, 0.0),
            "slow": lambda j: j / 4, "down": lambda j: -j / 4.0, "very large": lambda j: 200.0 * (j // 100)}


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("profile", PROFILES)
def test_climbing_scores(df, profile, d, dtype):
    """Weights that leave the range which the reference of earlier tiles gives them."""
    for n, G, block in ((2, 3, 1), (200, 1, 1), (200, 1, ALL)):
        b = pu.Batch(10, [430], [n], [(0, FULL)] * 2, G, d, dtype)
        b.q = (b.q.float() * 0.1).to(dtype)
        b.q[..., 0] = d ** 0.5
        p = torch.tensor(np.asarray(PROFILES[profile](np.arange(430 + n)), dtype=np.float64))
        for h in range(2):
            b.hist[0][h][0][:, 0] = p[:430].to(dtype)
            b.k_new[:, h, 0] = p[430:].to(dtype)
        repack(b)
        rows = sorted(set(range(0, n, 7)) | {n - 1})
        out, lse = run(df, b, block)
        pu.check(out, lse, b.reference(block, rows), dtype, d, "%s %d" % (profile, n), rows=rows)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["head-major", "wide"])
def test_layouts_of_the_new_tokens(df, kind, layout):
    n, G, block = KINDS[kind]
    b = pu.Batch(11, [77], [n], [(0, FULL), (5, 40)], G, 128, BF16)
    base, lse = run(df, b, block)

    def laid_out(t):
        t = t.to(DEV)
        if layout == "head-major":
            return t.transpose(0, 1).contiguous().transpose(0, 1)
        wide = torch.full((t.shape[0], t.shape[1] + 1, 2 * t.shape[2]), float("nan"), dtype=t.dtype, device=DEV)
        wide[:, 1:, 8:8 + t.shape[2]] = t
        return wide[:, 1:, 8:8 + t.shape[2]]
    out = laid_out(torch.full_like(base, 3.0))
    ls = torch.zeros_like(lse)
    ws = torch.empty(df.df_paged_workspace_bytes(2 * G, 2, 128, n), dtype=torch.uint8, device=DEV)
    df.df_paged_attn(laid_out(b.q), laid_out(b.k_new), laid_out(b.v_new), b.cache(df), b.cu, out, b.scale, block=block, max_new=n, lse_out=ls, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, base) and torch.equal(ls, lse)
    if layout == "wide":
        rest = out._base.clone()
        rest[:, 1:, 8:136] = float("nan")
        assert rest.isnan().all()


@pytest.mark.parametrize("kind", KINDS)
def test_rows_of_no_request_and_requests_cut_short(df, kind):
    n, G, block = KINDS[kind]
    b = pu.Batch(12, [40, 9], [n, n], [(0, FULL)], G, 64, FP16)
    base, lse = run(df, b, block)
    # five rows before the first request
    pad = lambda t: torch.cat([torch.full((5, *t.shape[1:]), float("nan"), dtype=t.dtype), t])
    b.q, b.k_new, b.v_new, b.cu = pad(b.q), pad(b.k_new), pad(b.v_new), b.cu + 5
    out, lse2 = run(df, b, block)
    assert torch.equal(out[5:], base) and torch.equal(lse2[:, 5:], lse) and (out[:5] == 7.0).all() and (lse2[:, :5] == 7.0).all()
    # requests count as far as max_new tokens
    short = n - 1
    out, lse2 = run(df, b, block, max_new=short)
    cut = pu.Batch(12, [40, 9], [n, n], [(0, FULL)], G, 64, FP16)
    keep = [i for r in range(2) for i in range(r * n, r * n + short)]
    cut.q, cut.k_new, cut.v_new, cut.cu, cut.new = cut.q[keep], cut.k_new[keep], cut.v_new[keep], ints([0, short, 2 * short]), [short, short]
    want, lse3 = run(df, cut, block)
    at = [5 + i for i in keep]
    assert torch.equal(out[at], want) and torch.equal(lse2[:, at], lse3)
    rest = [i for i in range(5 + 2 * n) if i not in at]
    assert (out[rest] == 7.0).all() and (lse2[:, rest] == 7.0).all()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024])
def test_every_page_size(df, page):
    for n, G, d, dtype in ((1, 2, 128, BF16), (70, 1, 64, FP16)):
        b = pu.Batch(page, [1100, 15], [n, n], [(0, FULL), (page + 3, 50)], G, d, dtype, page)
        out, lse = run(df, b, 1)
        pu.check(out, lse, b.reference(1), dtype, d, "page %d" % page)


@pytest.mark.parametrize("n,G,L", [(1, 1, 20001), (3, 8, 9000), (130, 1, 9000), (300, 2, 8600)])
def test_long_histories(df, n, G, L):
    """More tiles than are looked up at once, units that many workgroups share, rounds that begin anywhere."""
    b = pu.Batch(L + n, [L, 37], [n, 1], [(0, FULL)], G, 128, BF16, page=64)
    rows = sorted({0, n // 2, n - 1, n})
    out, lse = run(df, b, 1)
    pu.check(out, lse, b.reference(1, rows), BF16, 128, "history of %d" % L, rows=rows)
    again, _ = run(df, b, 1)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", KINDS)
def test_pages_far_into_a_pool(df, kind):
    """Rows of a pool of more than 2^32 bytes, where the last page lies and where an offset in 32 bits would wrap."""
    n, G, block = KINDS[kind]
    d, page = 128, 1024
    b = pu.Batch(13, [5000], [n], [(0, FULL)], G, d, BF16, page, spare=1)
    base, lse = run(df, b, block)
    used = b.table[0, 0, :5].tolist()
    n_pages = (1 << 32) // (page * d * 2) + 40
    far = [n_pages - 1, (1 << 32) // (page * d * 2), 5, n_pages - 2, (1 << 31) // (page * d * 2)]
    k, v = (torch.empty(n_pages, page, d, dtype=BF16, device=DEV) for _ in range(2))
    for small, big in zip(used, far):
        k[big], v[big] = b.k_pages[small], b.v_pages[small]
    b.k_pages, b.v_pages, b.free = k, v, torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    b.table[0, 0, :5] = ints(far)
    out, lse2 = run(df, b, block)
    assert torch.equal(out, base) and torch.equal(lse, lse2)
    rows = torch.randn(3, 1, d, device=DEV).to(BF16)
    slots = ints([[n_pages * page - 1], [(1 << 32) // (2 * d)], [-1]], torch.int64)
    df.df_paged_append(b.cache(df), rows, -rows, slots)
    torch.cuda.synchronize()
    for pool, want in ((k, rows), (v, -rows)):
        assert torch.equal(pool[-1, -1], want[0, 0]) and torch.equal(pool.view(-1, d)[(1 << 32) // (2 * d)], want[1, 0])


@pytest.mark.parametrize("B,H,n,G", [(1700, 10, 1, 2), (110, 20, 40, 1)])
def test_very_many_requests(df, B, H, n, G):
    """More heads than a workgroup notes in LDS, and more units than it looks at in one go."""
    lens = [(7 * i) % 21 for i in range(B)]
    b = pu.Batch(B, lens, [n if i % 5 else n // 2 for i in range(B)], [(0, FULL)] * (H - 1) + [(2, 9)], G, 64, BF16)
    rows = sorted(range(0, sum(b.new), 97))
    out, lse = run(df, b, 1)
    pu.check(out, lse, b.reference(1, rows), BF16, 64, "%d requests" % B, rows=rows)
    assert not out.isnan().any() and not (out == 7.0).all(-1).any()


# ---- all three together -----------------------------------------------------------------------------------------------------------

class Loop:
    """A serving loop on the device, and its tokens by position beside it."""

    def __init__(self, df, caps, B=3, G=1, d=64, dtype=BF16, page=16, n_pages=400, max_pages=60, seed=0):
        self.df, self.caps, self.B, self.H, self.G, self.d, self.dtype = df, caps, B, len(caps), G, d, dtype
        self.gen = torch.Generator().manual_seed(seed)
        order = np.random.default_rng(seed).permutation(n_pages).tolist()
        self.m = pu.Model(B, [caps] * B, n_pages, page, max_pages, order)
        nan = lambda: torch.full((n_pages, page, d), float("nan"), dtype=dtype, device=DEV)
        self.length, self.n_free, self.status = ints([0] * B), ints([n_pages]), ints([9])
        cap = ints(caps)
        self.cache = df.PagedCache(nan(), nan(), torch.full((B, self.H, max_pages), -3, dtype=torch.int32, device=DEV), self.length,
                                   cap[:, 0].contiguous(), cap[:, 1].contiguous(), ints(order), self.n_free)
        self.past = [[] for _ in range(B)]             # (k, v) [H, d] by position
        self.ws = torch.empty(df.df_paged_workspace_bytes(self.H * G, self.H, d, 200), dtype=torch.uint8, device=DEV)

    def tokens(self, total):
        rnd = lambda *s: torch.randn(*s, generator=self.gen).to(self.dtype)
        return rnd(total, self.H * self.G, self.d), rnd(total, self.H, self.d), rnd(total, self.H, self.d)

    def launch(self, q, k, v, cu, block, slots, out, lse, rel=None, stream=None, ws=None):
        """One step: attention of the new tokens, then their slots, then their rows."""
        df = self.df
        df.df_paged_attn(q, k, v, self.cache, cu, out, self.d ** -0.5, block=block, max_new=out.shape[0], lse_out=lse,
                         workspace=self.ws if ws is None else ws, stream=stream)
        df.df_page_map(self.cache, cu, slots, self.status, release=rel, stream=stream)
        df.df_paged_append(self.cache, k, v, slots, stream=stream)

    def expect(self, q, k, v, new, block):
        """The oracle of this step's attention."""
        b = object.__new__(pu.Batch)
        b.B, b.H, b.G, b.d, b.keys, b.scale = self.B, self.H, self.G, self.d, True, self.d ** -0.5
        b.caps, b.lens, b.new, b.q, b.k_new, b.v_new = [self.caps] * self.B, [len(x) for x in self.past], new, q, k, v
        stack = lambda r, h, x: torch.stack([p[x][h] for p in self.past[r]]) if self.past[r] else torch.zeros(0, self.d)
        b.hist = [[(stack(r, h, 0), stack(r, h, 1)) for h in range(self.H)] for r in range(self.B)]
        return b.reference(block)

    def advance(self, k, v, new, release=None):
        """The same on the oracle's side: slots of the new tokens."""
        slots = self.m.map(new, release)
        at = 0
        for r, n in enumerate(new):
            if release and release[r]:
                self.past[r] = []
            self.past[r] += [(k[at + i], v[at + i]) for i in range(n)]
            at += n
        return slots

    def agrees(self, slots, want):
        assert self.status.item() == self.df.DF_OK and slots[: len(want)].cpu().tolist() == want and (slots[len(want):] == -1).all()
        assert self.length.cpu().tolist() == self.m.len == [len(x) for x in self.past] and self.n_free.item() == len(self.m.free)


@pytest.mark.parametrize("G,d,dtype", [(1, 64, BF16), (3, 128, FP16)])
def test_a_loop_of_steps(df, G, d, dtype):
    """Prompts, pieces and single tokens; requests that end and are replaced."""
    loop = Loop(df, [(0, FULL), (4, 40), (0, 33), (0, 0)], G=G, d=d, dtype=dtype)
    steps = [([50, 0, 130], None, 1), ([1, 7, 1], None, 1), ([20, 20, 20], None, 20), ([1, 1, 1], None, 1), ([1, 64, 1], [0, 1, 0], ALL), ([1, 1, 1], None, 1),
             ([0, 0, 90], [1, 0, 1], 30), ([1, 1, 1], None, 1)]
    for i, (new, release, block) in enumerate(steps):
        q, k, v = loop.tokens(sum(new))
        if release:                                    # a request that begins has nothing behind it
            loop.df.df_page_map(loop.cache, ints([0] * 4), torch.empty(0, 4, dtype=torch.int64, device=DEV), loop.status, release=ints(release, torch.uint8))
            loop.advance(k, v, [0, 0, 0], release)
        ref = loop.expect(q, k, v, new, block)
        out, lse = torch.zeros(q.shape, dtype=dtype, device=DEV), torch.zeros(q.shape[1], q.shape[0], device=DEV)
        slots = torch.zeros(q.shape[0], 4, dtype=torch.int64, device=DEV)
        loop.launch(q.to(DEV), k.to(DEV), v.to(DEV), ints([0, *np.cumsum(new).tolist()]), block, slots, out, lse)
        torch.cuda.synchronize()
        pu.check(out, lse, ref, dtype, d, "step %d" % i)
        loop.agrees(slots, loop.advance(k, v, new))


def test_a_captured_step_is_replayed_while_requests_grow(df):
    """One graph serves every step of its shape: lengths and tables advance on the device.  Eager steps of other shapes go between, and a second graph."""
    loop = Loop(df, [(0, FULL), (4, 40)], G=2, d=128, seed=1)
    shapes = {"token": (6, 1), "piece": (120, 30)}
    graphs = {}
    for name, (rows, block) in shapes.items():
        buf = dict(q=torch.zeros(rows, 4, 128, dtype=BF16, device=DEV), k=torch.zeros(rows, 2, 128, dtype=BF16, device=DEV),
                   v=torch.zeros(rows, 2, 128, dtype=BF16, device=DEV), cu=ints([0] * 4), slots=torch.zeros(rows, 2, dtype=torch.int64, device=DEV),
                   out=torch.zeros(rows, 4, 128, dtype=BF16, device=DEV), lse=torch.zeros(4, rows, device=DEV))
        ws = torch.empty(df.df_paged_workspace_bytes(4, 2, 128, rows), dtype=torch.uint8, device=DEV)
        step = lambda: loop.launch(buf["q"], buf["k"], buf["v"], buf["cu"], block, buf["slots"], buf["out"], buf["lse"], ws=ws)
        step()                                         # no tokens: nothing moves
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs[name] = (g, buf, rows, block, ws)
    assert loop.length.tolist() == [0, 0, 0]
    for i, (name, new) in enumerate([("piece", [40, 70, 5]), ("token", [1, 1, 1]), ("token", [2, 0, 4]), ("eager", [9, 9, 9]), ("token", [1, 1, 1]),
                                     ("piece", [0, 100, 20]), ("token", [1, 1, 1]), ("eager", [33, 0, 1]), ("piece", [1, 1, 1]), ("token", [0, 0, 1])]):
        q, k, v = loop.tokens(sum(new))
        cu = ints([0, *np.cumsum(new).tolist()])
        if name == "eager":
            block, n = 1, sum(new)
            buf = dict(out=torch.zeros(n, 4, 128, dtype=BF16, device=DEV), lse=torch.zeros(4, n, device=DEV), slots=torch.zeros(n, 2, dtype=torch.int64, device=DEV))
            ref = loop.expect(q, k, v, new, block)
            loop.launch(q.to(DEV), k.to(DEV), v.to(DEV), cu, block, buf["slots"], buf["out"], buf["lse"])
        else:
            g, buf, rows, block, _ = graphs[name]
            n = sum(new)
            for x, t in (("q", q), ("k", k), ("v", v)):
                buf[x].fill_(float("nan"))
                buf[x][:n] = t.to(DEV)
            buf["cu"].copy_(cu)
            ref = loop.expect(q, k, v, new, block)
            g.replay()
        torch.cuda.synchronize()
        pu.check(buf["out"], buf["lse"], ref, BF16, 128, "%d: %s" % (i, name))
        loop.agrees(buf["slots"], loop.advance(k, v, new))


def test_a_step_on_another_stream(df):
    loop = Loop(df, [(0, FULL), (4, 40)], seed=2)
    side = torch.cuda.Stream()
    for i, new in enumerate(([30, 80, 1], [1, 1, 1], [64, 64, 64])):
        q, k, v = loop.tokens(sum(new))
        ref = loop.expect(q, k, v, new, 1)
        dev = [t.to(DEV) for t in (q, k, v)]
        cu = ints([0, *np.cumsum(new).tolist()])
        out, lse, slots = torch.zeros_like(dev[0]), torch.zeros(2, q.shape[0], device=DEV), torch.zeros(q.shape[0], 2, dtype=torch.int64, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        if i == 1:
            with torch.cuda.stream(side):
                loop.launch(*dev, cu, 1, slots, out, lse)
        else:
            loop.launch(*dev, cu, 1, slots, out, lse, stream=side if i else side.cuda_stream)
        side.synchronize()
        pu.check(out, lse, ref, BF16, 64, "step %d" % i)
        loop.agrees(slots, loop.advance(k, v, new))


def test_two_calls_at_once(df):
    """Calls on two streams, each with a workspace of its own, and two captured ones replayed beside each other: as one after the other."""
    calls = []
    for seed, (lens, new, G, block) in enumerate([([4000, 900], [1, 1], 4, 1), ([700, 0, 1200], [130, 64, 1], 1, 40)]):
        b = pu.Batch(20 + seed, lens, new, [(0, FULL), (8, 300)], G, 128, BF16)
        want, lse = run(df, b, block)
        q, k, v = b.q.to(DEV), b.k_new.to(DEV), b.v_new.to(DEV)
        ws = torch.empty(df.df_paged_workspace_bytes(2 * G, 2, 128, max(new)), dtype=torch.uint8, device=DEV)
        out, ls, cache, stream = torch.empty_like(want), torch.empty_like(lse), b.cache(df), torch.cuda.Stream()
        call = lambda b=b, q=q, k=k, v=v, ws=ws, out=out, ls=ls, cache=cache, block=block, new=new: df.df_paged_attn(
            q, k, v, cache, b.cu, out, b.scale, block=block, max_new=max(new), lse_out=ls, workspace=ws)
        calls.append((call, stream, out, ls, want, lse))
    torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        for _, _, out, ls, want, lse in calls:
            assert torch.equal(out, want) and torch.equal(ls, lse)
            out.fill_(7.0)
            ls.fill_(7.0)
        torch.cuda.synchronize()
    for _ in range(5):
        for call, stream, *_ in calls:
            with torch.cuda.stream(stream):
                call()
    same()
    graphs = []
    for call, stream, *_ in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call()
        graphs.append(g)
    same_first = [c[2].clone() for c in calls]
    assert all((x == 7.0).all() for x in same_first)        # captured, not run
    for _ in range(3):
        for g, (_, stream, *_rest) in zip(graphs, calls):
            with torch.cuda.stream(stream):
                g.replay()
        same()


@pytest.mark.parametrize("kind", KINDS)
def test_batches_of_nothing(df, kind):
    """No request has a new token: nothing is written, and the map changes nothing."""
    n, G, block = KINDS[kind]
    b = pu.Batch(16, [60, 5], [n, n], [(0, FULL)], G, 64, BF16)
    for at in (0, 3, 2 * n):
        b.cu = ints([at] * 3)
        out, lse = run(df, b, block)
        assert (out == 7.0).all() and (lse == 7.0).all()
        slots, status = torch.zeros(2 * n, 1, dtype=torch.int64, device=DEV), ints([5])
        before = [x.clone() for x in (b.table, b.length, b.free, b.n_free)]
        df.df_page_map(b.cache(df), b.cu, slots, status)
        torch.cuda.synchronize()
        assert status.item() == df.DF_OK and (slots == -1).all()
        assert all(torch.equal(x, y) for x, y in zip(before, (b.table, b.length, b.free, b.n_free)))


def test_one_request_is_the_dense_call(df):
    """A single request whose new tokens all see each other: what df_attn_fwd computes from packed histories."""
    caps = [(0, FULL), (20, 60), (0, 40), (0, 0)]
    b = pu.Batch(14, [150], [140], caps, 1, 128, BF16)
    b.sees_all = [pu.held_positions(150, s, w) for s, w in caps]
    out, lse = run(df, b, 1 << 20)
    # later tokens of one block do not push history out: `first` is 0 for all
    off = np.concatenate([[0], np.cumsum([len(x) for x in b.sees_all])]).tolist()
    k0, v0 = (torch.cat([b.hist[0][h][x][at] for h, at in enumerate(b.sees_all)]).to(DEV) for x in range(2))
    dense, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    ws = torch.empty(df.df_attn_workspace_bytes(4, 128, 140), dtype=torch.uint8, device=DEV)
    df.df_attn_fwd(b.q.to(DEV), b.k_new.to(DEV), b.v_new.to(DEV), k0, v0, off, None, dense, b.scale, lse_out=lse2, workspace=ws)
    torch.cuda.synchronize()
    tol, tol_lse = pu.bounds(b.reference(1 << 20), BF16, 128)
    assert (np.abs((out.double() - dense.double()).cpu().numpy()) <= 2 * tol).all()
    assert (np.abs((lse.double() - lse2.double()).cpu().numpy()) <= 2 * tol_lse).all()


@pytest.mark.parametrize("n", [1, 40])
def test_native_and_python_marshalling_make_the_same_calls(df, monkeypatch, n):
    b = pu.Batch(15, [60, 7], [n, n], [(0, FULL), (3, 20)], 2, 64, BF16)

    def results():
        cache = df.PagedCache(b.k_pages.clone(), b.v_pages.clone(), b.table.clone(), b.length.clone(), b.sink, b.win, b.free.clone(), b.n_free.clone())
        out = [*b.run(df, 1, cache=cache), *b.run(df, 1, cache=cache, lse=False, stream=torch.cuda.current_stream())[:1]]
        slots, status = torch.zeros(2 * n, 2, dtype=torch.int64, device=DEV), ints([5])
        length, n_free = ints([0, 0]), ints([0])
        errors = []
        for release, more in ((None, {}), (ints([0, 1], torch.uint8), dict(stream=0)), (None, dict(len_out=length, n_free_out=n_free))):
            df.df_page_map(cache, b.cu, slots, status, release=release, **more)
            df.df_paged_append(cache, b.k_new.to(DEV), b.v_new.to(DEV), slots, stream=more.get("stream"))
            out += [slots.clone(), status.clone(), cache.length.clone(), cache.n_free.clone()]
        q, o = b.q.to(DEV), torch.zeros(2 * n, 4, 64, dtype=BF16, device=DEV)
        ws = torch.empty(1 << 27, dtype=torch.uint8, device=DEV)
        df.df_paged_attn(q, None, None, cache, b.cu, o, 0.125, workspace=ws)
        for call in (lambda: df.df_paged_attn(q, q, None, cache, b.cu, o, 0.125, workspace=ws), lambda: df.df_paged_attn(q, q, q, cache, b.cu, o, 0.125, workspace=ws),
                     lambda: df.df_paged_attn(q, None, None, cache, b.cu[:1], o, 0.125, workspace=ws),
                     lambda: df.df_paged_attn(q, None, None, cache, b.cu, o[:1], 0.125, workspace=ws),
                     lambda: df.df_paged_attn(q.half(), None, None, cache, b.cu, o, 0.125, workspace=ws),
                     lambda: df.df_paged_attn(q, None, None, cache, b.cu, o, 0.125, lse_out=o, workspace=ws),
                     lambda: df.df_paged_append(cache, q, q, slots), lambda: df.df_paged_append(cache, b.k_new.to(DEV), b.k_new.to(DEV)[:, :1], slots),
                     lambda: df.df_page_map(cache, b.cu, slots.int(), status), lambda: df.df_page_map(cache, b.cu, slots, status, release=b.cu),
                     lambda: df.df_page_map(cache, b.cu, slots, status, len_out=n_free)):
            with pytest.raises(ValueError) as e:
                call()
            errors.append(str(e.value))
        for call in (lambda: df.df_paged_attn(q, None, None, cache, b.cu, o, 0.125), lambda: df.df_paged_attn(q, None, None, cache, b.cu, o, -1.0, workspace=ws),
                     lambda: df.df_paged_attn(q, None, None, cache, b.cu, o, 0.125, block=0, workspace=ws),
                     lambda: df.df_paged_attn(q, None, None, cache, b.cu, o, 0.125, max_new=0, workspace=ws)):
            with pytest.raises(df.DfError) as e:
                call()
            errors.append((e.value.status, str(e.value)))
        torch.cuda.synchronize()
        return [*out, o, cache.k_pages, cache.v_pages, cache.block_table], errors

    native = df._marshal()
    assert native
    monkeypatch.setattr(df, "_native", native)
    tensors, errors = results()
    monkeypatch.setattr(df, "_native", False)
    for x, y in zip(tensors, results()[0]):
        assert (x is None and y is None) or torch.equal(x.nan_to_num() if x.is_floating_point() else x, y.nan_to_num() if y.is_floating_point() else y)
    assert errors == results()[1]
