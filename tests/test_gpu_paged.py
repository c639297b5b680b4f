"""df_page_map, df_paged_append and df_paged_attn against the plain model of paged_util, through the C ABI."""
import numpy as np
import pytest
import torch

from tests import paged_util as pu
from tests.paged_util import FULL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def df():
    from paper_2601_20499_amd import binding
    return binding


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


# ---- block tables and slot maps -----------------------------------------------------------------------------------------------

class Device:
    """A paged cache on the device beside the model."""

    def __init__(self, df, B, caps, n_pages, page, max_pages, seed=0, d=64, dtype=BF16, per_request=True):
        rng = np.random.default_rng(seed)
        order = rng.permutation(n_pages).tolist()
        self.m = pu.Model(B, caps, n_pages, page, max_pages, order)
        H = len(caps[0])
        self.table = torch.full((B, H, max_pages), -7, dtype=torch.int32, device=DEV)
        self.length, self.n_free, self.free = ints([0] * B), ints([n_pages]), ints(order)
        cap = ints(caps if per_request else caps[0])
        self.k = torch.full((n_pages, page, d), 9.0, dtype=dtype, device=DEV)
        self.v = torch.full((n_pages, page, d), 9.0, dtype=dtype, device=DEV)
        self.cache = df.PagedCache(self.k, self.v, self.table, self.length, cap[..., 0].contiguous(), cap[..., 1].contiguous(), self.free,
                                   self.n_free)
        self.status = ints([99])

    def step(self, df, new, release=None, pad=0):
        """One df_page_map; device and model have to agree in everything.  Returns the device's slot map."""
        m = self.m
        total = sum(new) + pad
        slots = torch.full((total, m.H), 123456, dtype=torch.int64, device=DEV)
        cu = ints(np.concatenate([[0], np.cumsum(new)]).tolist())
        before = self.table.cpu().clone()
        rel = None if release is None else ints(release, torch.uint8)
        df.df_page_map(self.cache, cu, slots, self.status, release=rel)
        torch.cuda.synchronize()
        want = m.map(new, release)
        table = self.table.cpu()
        if want is None:
            assert self.status.item() == df.DF_ERR_RANGE and (slots == -1).all() and torch.equal(table, before)
        else:
            assert self.status.item() == df.DF_OK
            assert slots.cpu().tolist() == want + [[-1] * m.H] * pad
            for b in range(m.B):
                for h in range(m.H):
                    own = m.pages[b][h]
                    assert table[b, h, :len(own)].tolist() == own, (b, h)
                    if not (release and release[b]):
                        assert torch.equal(table[b, h, len(own):], before[b, h, len(own):]), (b, h)
        assert self.length.cpu().tolist() == m.len and self.n_free.item() == len(m.free)
        assert self.free[:len(m.free)].cpu().tolist() == m.free
        return slots


@pytest.mark.parametrize("seed", range(6))
def test_map_against_the_model(df, seed):
    """Requests that grow by nothing, single tokens and chunks past their windows, end and are replaced; some steps do not fit."""
    rng = np.random.default_rng(seed)
    B, H, page = int(rng.integers(1, 7)), int(rng.integers(1, 6)), int(2 ** rng.integers(4, 8))
    pick = lambda: [(0, 0), (0, int(rng.integers(1, 200))), (int(rng.integers(1, 100)), 0), (int(rng.integers(1, 60)), int(rng.integers(1, 150))),
                    (0, FULL), (FULL, FULL)][rng.integers(6)]
    caps = [[pick() for _ in range(H)] for _ in range(B)]
    dev = Device(df, B, caps, int(rng.integers(20, 120)), page, int(rng.integers(4, 12)), seed)
    for step in range(25):
        new = [int(x) for x in rng.choice([0, 0, 1, 1, 2, 17, 64, 150, 333], size=B)]
        release = [int(rng.random() < 0.15) * int(rng.integers(1, 256)) for _ in range(B)] if step % 3 == 2 else None
        dev.step(df, new, release, pad=int(rng.integers(0, 3)))


def test_map_many_heads_and_many_slots(df):
    """More (request, head) entries than threads, and more slots than one workgroup writes; one head that takes hundreds of pages."""
    rng = np.random.default_rng(5)
    caps = [[[(0, FULL), (3, 40), (0, 0), (16, 0)][(b + h) % 4] for h in range(40)] for b in range(70)]
    dev = Device(df, 70, caps, 30000, 16, 400, 1)
    dev.step(df, [int(x) for x in rng.integers(0, 30, size=70)])
    dev.step(df, [5000] + [1] * 69)
    dev.step(df, [1] * 70, release=[int(b % 3 == 0) for b in range(70)])
    dev.step(df, [0] * 70, release=[1] * 70)
    assert dev.n_free.item() == 30000


def test_map_all_or_nothing(df):
    """A step that needs one page too many takes none; the same step fits once a request has ended."""
    dev = Device(df, 2, [[(0, FULL)]] * 2, 4, 16, 4)
    dev.step(df, [33, 16])
    dev.step(df, [1, 1])                                     # 0 pages left: nothing fits
    assert dev.status.item() == df.DF_ERR_RANGE
    dev.step(df, [1, 5], release=[0, 1])
    assert dev.status.item() == df.DF_OK
    dev.step(df, [40, 0], release=[0, 1])                    # 5 pages of a table of 4
    assert dev.status.item() == df.DF_ERR_RANGE


@pytest.mark.parametrize("spoil", ["len", "cu_falls", "cu_beyond", "cu_negative", "n_free", "n_free_negative", "cap", "free_id", "held_id"])
def test_map_reports_arrays_out_of_range(df, spoil):
    dev = Device(df, 2, [[(0, FULL), (8, 8)]] * 2, 40, 16, 4)
    dev.step(df, [20, 20])
    cu, total, release = [0, 3, 6], 6, None
    if spoil == "len":
        dev.length[1] = -1
    if spoil == "cu_falls":
        cu = [0, 4, 3]
    if spoil == "cu_beyond":
        cu = [0, 3, 7]
    if spoil == "cu_negative":
        cu = [-1, 3, 6]
    if spoil == "n_free":
        dev.n_free.fill_(41)
    if spoil == "n_free_negative":
        dev.n_free.fill_(-1)
    if spoil == "cap":
        dev.cache.sink_cap[0, 1] = -5
    if spoil == "free_id":
        cu, total = [0, 20, 40], 40
        dev.free[dev.n_free.item() - 1] = 40
    if spoil == "held_id":
        release = ints([1, 0], torch.uint8)
        dev.table[0, 0, 1] = 1 << 20
    state = [t.clone() for t in (dev.table, dev.length, dev.n_free, dev.free)]
    slots = torch.zeros(total, 2, dtype=torch.int64, device=DEV)
    df.df_page_map(dev.cache, ints(cu), slots, dev.status, release=release)
    torch.cuda.synchronize()
    assert dev.status.item() == df.DF_ERR_RANGE and (slots == -1).all()
    for was, now in zip(state, (dev.table, dev.length, dev.n_free, dev.free)):
        assert torch.equal(was, now)


# ---- rows into pages ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,dtype,layout", [(128, BF16, "thd"), (64, FP16, "htd"), (128, FP16, "wide")])
def test_append_writes_the_slots_and_nothing_else(df, d, dtype, layout):
    caps = [[(5, 40), (0, 0), (0, FULL)], [(0, 17), (33, 0), (1, 1)]]
    dev = Device(df, 2, caps, 40, 16, 8, 3, d=d, dtype=dtype)
    g = torch.Generator().manual_seed(1)
    k_want, v_want = dev.k.cpu().clone(), dev.v.cpu().clone()
    for new in ([7, 0], [1, 1], [60, 45], [0, 3]):
        slots = dev.step(df, new, pad=2)
        total = slots.shape[0]
        k, v = (torch.randn(total, 3, d, generator=g).to(dtype) for _ in range(2))
        if layout == "htd":
            kd, vd = (x.permute(1, 0, 2).contiguous().to(DEV).permute(1, 0, 2) for x in (k, v))
        elif layout == "wide":
            kd, vd = (torch.cat([x, x], 2).to(DEV)[:, :, :d] for x in (k, v))
        else:
            kd, vd = k.to(DEV), v.to(DEV)
        df.df_paged_append(dev.cache, kd, vd, slots)
        torch.cuda.synchronize()
        s = slots.cpu()
        k_want.view(-1, d)[s[s >= 0]] = k[s >= 0]
        v_want.view(-1, d)[s[s >= 0]] = v[s >= 0]
        assert torch.equal(dev.k.cpu(), k_want) and torch.equal(dev.v.cpu(), v_want)


def test_append_skips_slots_outside_the_pool(df):
    dev = Device(df, 1, [[(0, FULL)]], 2, 16, 2)
    slots = ints([[-1], [32], [1 << 40], [-(1 << 40)], [31]], torch.int64)
    k = torch.randn(5, 1, 64, device=DEV).to(BF16)
    df.df_paged_append(dev.cache, k, k, slots)
    torch.cuda.synchronize()
    assert torch.equal(dev.k.view(-1, 64)[31], k[4, 0]) and (dev.k.view(-1, 64)[:31] == 9.0).all()


# ---- attention ------------------------------------------------------------------------------------------------------------------

MIXED = [(7, 50), (0, 0), (40, 0), (0, 33), (0, FULL), (64, 64)]
CASES = [
    # name, lens, new, caps, G, d, dtype, page, block, keys
    ("one token, nothing behind it", [0], [1], [(0, FULL)], 1, 64, BF16, 16, 1, True),
    ("one token, one behind it", [1], [1], [(0, FULL)], 1, 128, BF16, 16, 1, True),
    ("tokens, odd lengths, grouped heads", [0, 1, 15, 16, 17, 31, 33, 64, 127, 300, 777], [1] * 11, [(0, FULL)] * 3, 4, 128, BF16, 16, 1, True),
    ("tokens d 64 fp16", [5, 63, 64, 65, 1000], [1] * 5, [(0, FULL)] * 2, 7, 64, FP16, 32, 1, True),
    ("tokens, some requests have none", [9, 200, 40, 0, 12], [1, 0, 1, 0, 1], MIXED, 1, 128, BF16, 16, 1, True),
    ("tokens, 17 to 32 rows", [300, 45, 0], [5, 3, 4], MIXED, 5, 128, BF16, 16, 1, True),
    ("tokens, 32 rows, fp16, d 64", [513, 64], [4, 4], [(0, FULL), (3, 90)], 8, 64, FP16, 64, 2, True),
    ("drafted tokens, windows cut inside the chunk", [100, 3, 0, 57], [12, 7, 16, 1], [(0, 5), (2, 3), (0, 1), (4, 9)], 1, 128, BF16, 16, 1, True),
    ("one long history", [5000], [2], [(0, FULL)] * 2, 2, 128, BF16, 128, 1, True),
    ("looking back only, some see nothing", [0, 30, 0, 200], [3, 3, 1, 40], MIXED, 1, 128, BF16, 16, 1, False),
    ("few rows, looking back only", [0, 30, 0, 200], [3, 3, 1, 4], MIXED, 1, 64, FP16, 16, 2, False),
    ("prompt from nothing", [0], [200], [(0, FULL)] * 2, 1, 128, BF16, 16, 1, True),
    ("prompt pieces, ragged, one single token", [0, 130, 77, 5], [150, 33, 1, 64], [(0, FULL)] * 2, 4, 128, BF16, 16, 1, True),
    ("pieces, every head type, token by token", [150, 0, 64, 29], [90, 70, 0, 131], MIXED, 1, 128, BF16, 32, 1, True),
    ("frames, every head type", [150, 0, 300], [99, 66, 33], MIXED, 1, 64, FP16, 16, 33, True),
    ("whole chunk, every head type, wrapped rings", [401, 129], [100, 130], MIXED, 2, 128, BF16, 64, 1 << 30, True),
    ("whole chunk, d 64", [100, 1], [190, 64], MIXED, 1, 64, BF16, 16, 500, True),
    ("frames against windows shorter than a chunk", [500, 20], [120, 121], [(0, 37), (11, 40), (0, 64), (200, 10)], 1, 128, FP16, 16, 40, True),
    ("pages longer than a tile", [700, 90], [80, 40], MIXED, 3, 128, BF16, 1024, 1, True),
    ("many rows of few tokens", [90, 10], [3, 2], [(0, FULL)], 64, 64, BF16, 16, 1, True),
]


@pytest.mark.parametrize("case", CASES, ids=[c[0].replace(" ", "_") for c in CASES])
def test_attention_against_the_model(df, case):
    name, lens, new, caps, G, d, dtype, page, block, keys = case
    b = pu.Batch(len(name), lens, new, caps, G, d, dtype, page, keys)
    out, lse = b.run(df, block, extra_rows=2)
    torch.cuda.synchronize()
    pu.check(out, lse, b.reference(block), dtype, d, name)
    n = sum(new)
    assert (out[n:] == 7.0).all() and (lse[:, n:] == 7.0).all()          # rows of no request
    again, lse2 = b.run(df, block, extra_rows=2)                       # bit for bit the same, without a log-sum-exp too
    only, _ = b.run(df, block, lse=False, extra_rows=2)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(lse, lse2) and torch.equal(out, only)
