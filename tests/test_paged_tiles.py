"""The asm statements of df_paged_tiles.inc: what is committed is what the generator writes, and an interpreter that knows registers by what
they hold runs two tiles of each statement: every product takes the operands that it should, from reads that have landed, and the
waits and wait states are there."""
import os
import re
import sys

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_20499_amd", "csrc")
sys.path.insert(0, CSRC)
import gen_paged_tiles as gen  # noqa: E402

STATEMENTS = [(D, fp16) for D in (128, 64) for fp16 in (False, True)]


def test_the_include_is_what_the_generator_writes():
    with open(gen.OUT) as f:
        assert f.read() == gen.text()


def lines_of(D, fp16):
    text = gen.statement(D, fp16)
    return [x for x in re.findall(r'"(.*?)\\n\\t"', text)]


def regs(x):
    m = re.match(r"([vs])\[(\d+):(\d+)\]$", x)
    if m:
        return [f"{m[1]}{i}" for i in range(int(m[2]), int(m[3]) + 1)]
    return [x]


def run(lines, D, start, tiles, held=()):
    """Interprets from label `start` on until `tiles` tiles are done; returns what registers hold and a trace.  `held`: more registers at the start."""
    rowb, tile_bytes = 2 * D, gen.KT * 2 * D
    value, age, written_by = {}, {}, {}
    for (ks, qb), r in gen.Q.items():
        if ks < D // 32:
            for v in range(4):
                value[f"v{r + v}"] = ("q", ks, qb)
    for (db, qb), r in gen.O.items():
        if db < D // 16:
            for v in range(4):
                value[f"v{r + v}"] = ("o", db, qb, ())
    value["%[l0]"], value["%[l1]"] = ("l", 0, ()), ("l", 1, ())
    value.update(held)
    pending = []                                     # reads on their way: (registers, what)
    dma = 0
    clock = 0
    pc = lines.index(f"{start}:")
    buf = int(start[6])
    done, n = 0, tiles
    trace = dict(brought=[], barriers=0)
    label = {x[:-1]: i for i, x in enumerate(lines) if x.endswith(":")}
    m0 = None
    m0_at = -9

    def use(r, by):
        assert r in value, (r, by)
        assert not any(r in p[0] for p in pending), (r, "read before it has landed", by)
        if written_by.get(r) == "product" and by != "product":
            assert clock - age[r] >= 8, (r, "wait states behind a product", clock - age[r])
        if written_by.get(r) == "vector" and by == "product":
            assert clock - age[r] >= 3, (r, "wait states in front of a product")
        if written_by.get(r) == "exp":
            assert clock - age[r] >= 2, (r, "exponential used at once")
        return value[r]

    def put(r, what, by):
        assert not any(r in p[0] for p in pending), (r, "written under a read")
        value[r], age[r], written_by[r] = what, clock, by

    while True:
        x = lines[pc]
        pc += 1
        if x.endswith(":"):
            continue
        op, _, rest = x.partition(" ")
        args = [a.strip() for a in re.split(r",(?![^\[]*\])", rest)]
        if op == "s_waitcnt":
            m = re.search(r"lgkmcnt\((\d+)\)", rest)
            if m:
                while len(pending) > int(m[1]):
                    pending.pop(0)
            if "vmcnt(0)" in rest:
                dma = 0
            continue
        clock += 1 + (int(rest) if op == "s_nop" else 0)
        if op == "s_barrier":
            assert dma == 0 and not pending, "all reads and loads are waited for before the barrier"
            trace["barriers"] += 1
        elif op in ("s_nop", "s_mov_b32", "s_add_i32", "s_mul_hi_u32", "s_mul_i32", "s_addc_u32", "v_readlane_b32", "s_sub_i32", "s_cmp_eq_u32", "s_setprio"):
            if op == "s_sub_i32":
                n -= 1
        elif op == "s_add_u32":
            if args[0] == "m0":
                assert args[1] == "%[to]"
                m0, m0_at = int(args[2], 0), clock
        elif op == "buffer_load_dwordx4":
            assert clock - m0_at >= 2, "an instruction between m0 and the load"
            which = args[0][2]
            assert args[1] == ("s[64:67]" if which == "k" else "s[68:71]") and rest.endswith("offen lds")
            trace["brought"].append((args[0], m0))
            dma += 1
        elif op.startswith("ds_read"):
            m = re.match(r"(.*) offset:(\d+)$", rest)
            d, a = [y.strip() for y in m[1].split(",")]
            what = (op, a, int(m[2]))
            for r in regs(d):
                assert not any(r in p[0] for p in pending)
                value[r], age[r], written_by[r] = what, clock, "read"
            pending.append((regs(d), what))
        elif op.startswith("v_mfma"):
            d, a, b, c = [regs(y) for y in args]
            wa = [use(r, "product") for r in a]
            wb = [use(r, "product") for r in b]
            if c == ["0"]:
                acc = ()
            else:
                assert c == d
                acc = use(d[0], "product")[-1]
                assert len({use(r, "product") for r in d}) == 1
            key = value[d[0]][:-1] if c != ["0"] else ("s", d[0])
            term = (tuple(dict.fromkeys(wa)), tuple(dict.fromkeys(wb)))
            for r in d:
                put(r, (*key, acc + (term,)), "product")
        elif op == "v_fma_f32":
            assert args[2] == "%[c]" and args[3] in ("%[nm0]", "%[nm1]")
            s = use(args[1], "vector")
            put(args[0], ("e", args[1], s[-1], int(args[3][4])), "vector")
        elif op == "v_exp_f32":
            w = use(args[1], "vector")
            assert w[0] == "e"
            put(args[0], ("w", *w[1:]), "exp")
        elif op == "v_add_f32":
            terms = ()
            for a in args[1:]:
                w = use(a, "vector")
                terms += w[-1] if w[0] in ("sum", "l") else (w,)
            put(args[0], (("l", int(args[0][3])) if args[0].startswith("%[l") else ("sum",)) + (terms,), "vector")
        elif op.startswith("v_cvt_pk"):
            put(args[0], ("p", use(args[1], "vector"), use(args[2], "vector")), "vector")
        elif op == "v_cmp_nge_f32":
            use(args[2], "vector")
        elif op == "s_cbranch_vccnz":
            assert args[0] in ([f".Ldf_over{h}_%=" for h in range(2)])
            if args[0] == ".Ldf_over1_%=":
                trace.setdefault("before_second", dict(value))
        elif op == "s_cbranch_scc1":
            if n == 0:
                pc = label[args[0]]
        elif op == "s_cbranch_scc0":
            if n:
                pc = label[args[0]]
        elif op == "s_branch":
            pc = label[args[0]]
        else:
            raise AssertionError(x)
        if pc == len(lines):
            assert not pending
            return value, trace


@pytest.mark.parametrize("D,fp16", STATEMENTS)
@pytest.mark.parametrize("buf", [0, 1])
def test_two_tiles(D, fp16, buf):
    lines = lines_of(D, fp16)
    value, trace = run(lines, D, f".Ldf_b{buf}_%=", 2)
    rowb, tile_bytes, loads = 2 * D, gen.KT * 2 * D, D // 32
    assert trace["barriers"] == 2
    # the tile behind the first goes into the other buffer, K and V, every load to its KB
    want = []
    for t in range(2):
        to = ((buf + t + 1) % 2) * 2 * tile_bytes
        want += [(f"%[ko{i}]", to + 1024 * i) for i in range(loads)] + [(f"%[vo{i}]", to + tile_bytes + 1024 * i) for i in range(loads)]
    assert trace["brought"] == want

    def k_at(t, kb, ks):
        return ("ds_read_b128", f"%[k{ks}]", ((buf + t) % 2) * 2 * tile_bytes + (32 * (kb // 2) + 4 * (kb % 2)) * rowb)

    def v_at(t, h, db, u):
        return ("ds_read_b64_tr_b16", f"%[v{db}]", ((buf + t) % 2) * 2 * tile_bytes + (32 * h + 4 * u) * rowb)

    def score(t, kb, qb):
        return tuple(((k_at(t, kb, ks),), (("q", ks, qb),)) for ks in range(D // 32))

    def weight(t, kb, qb, v):
        return ("w", f"v{gen.S[kb, qb] + v}", score(t, kb, qb), qb)

    for qb in range(2):
        for db in range(D // 16):
            terms = []
            for t in range(2):
                for h in range(2):
                    p = tuple(("p", weight(t, 2 * h + u, qb, 2 * i), weight(t, 2 * h + u, qb, 2 * i + 1)) for u in range(2) for i in range(2))
                    terms.append(((v_at(t, h, db, 0), v_at(t, h, db, 1)), p))
            for v in range(4):
                assert value[f"v{gen.O[db, qb] + v}"] == ("o", db, qb, tuple(terms)), (db, qb)
        # the sums: every weight of both tiles once
        got = sorted(map(str, value[f"%[l{qb}]"][-1]))
        assert got == sorted(str(weight(t, kb, qb, v)) for t in range(2) for kb in range(4) for v in range(4))
    # where the second half is left, outputs and sums hold the first half only
    first = trace["before_second"]
    for (db, qb), r in gen.O.items():
        if db < D // 16:
            assert len(first[f"v{r}"][-1]) == 1
    assert all(w[1] in {f"v{gen.S[kb, qb] + v}" for kb in range(2) for v in range(4)} for qb in range(2) for w in first[f"%[l{qb}]"][-1])


@pytest.mark.parametrize("D,fp16", STATEMENTS)
def test_the_statement_says_what_it_writes(D, fp16):
    text = gen.statement(D, fp16)
    body, rest = text.split("\n      : ", 1)
    written = set()
    for x in re.findall(r'"(.*?)\\n\\t"', body):
        m = re.match(r"(v_(?!cmp)\w+|ds_read\w+)\s+([^,]+),", x)
        if m:
            written |= set(regs(m[2]))
    said = {f"v{i}" for i in re.findall(r'"v(\d+)"', rest)}
    for a, b in re.findall(r'"\+\{v\[(\d+):(\d+)\]\}"', rest):
        said |= {f"v{i}" for i in range(int(a), int(b) + 1)}
    fixed = {r for r in written if r.startswith("v")}
    assert fixed <= said
    # whatever way the statement ends, the wave's priority is the ordinary one again
    assert re.findall(r'"(.*?)\\n\\t"', body)[-4:] == [".Ldf_end_%=:", "s_setprio 0", "s_nop 7", "s_nop 7"]
    queries = {f"v{i}" for a, b in re.findall(r'"\{v\[(\d+):(\d+)\]\}"', rest) for i in range(int(a), int(b) + 1)}
    assert queries and not queries & (said | fixed)


@pytest.mark.parametrize("second", [False, True])
@pytest.mark.parametrize("D,fp16", STATEMENTS)
def test_a_product_by_itself(D, fp16, second):
    """S^T of all four blocks of keys, and O^T plus both halves' products."""
    text = gen.one_product(D, fp16, second)
    lines = ["s_begin:", *re.findall(r'"(.*?)\\n\\t"', text)]
    assert lines[-2:] == ["s_nop 7", "s_nop 7"] and all(("_f16 v" in x) == fp16 for x in lines if "mfma" in x)
    P = {f"v{gen.P[h, qb] + v}": ("weights", h, qb) for h in range(2) for qb in range(2) for v in range(4)}
    value, _ = run([".Ldf_b0_%=:", *lines[1:]], D, ".Ldf_b0_%=", 1, P if second else ())
    rowb = 2 * D
    for qb in range(2):
        if second:
            for db in range(D // 16):
                terms = tuple((tuple(("ds_read_b64_tr_b16", f"%[v{db}]", (32 * h + 4 * u) * rowb) for u in range(2)), (("weights", h, qb),)) for h in range(2))
                for v in range(4):
                    assert value[f"v{gen.O[db, qb] + v}"] == ("o", db, qb, terms)
        else:
            for kb in range(4):
                terms = tuple(((("ds_read_b128", f"%[k{ks}]", (32 * (kb // 2) + 4 * (kb % 2)) * rowb),), (("q", ks, qb),)) for ks in range(D // 32))
                for v in range(4):
                    assert value[f"v{gen.S[kb, qb] + v}"][-1] == terms
    # every register that is written is an output or said to be
    said = {f"v{i}" for i in re.findall(r'"v(\d+)"', text)}
    for a, b in re.findall(r'"(?:\+|=&)\{v\[(\d+):(\d+)\]\}"', text):
        said |= {f"v{i}" for i in range(int(a), int(b) + 1)}
    for x in lines:
        m = re.match(r"(v_mfma\w+|ds_read\w+)\s+(v\[\d+:\d+\]),", x)
        assert not m or set(regs(m[2])) <= said
