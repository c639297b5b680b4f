#!/usr/bin/env python3
"""Writes df_paged_tiles.inc: the loop of df_paged_many_kernel over whole tiles that all rows of a wave see, one asm statement per type
and head dimension.

A tile is 64 keys in two halves h of 32.  A wave's 32 rows go through it in four phases:

    S(0) = K(0) Q^T                              matrix core alone
    S(1) = K(1) Q^T    beside    P(0), sums      P = 2^(c s - m c)
    O += V(0) P(0)     beside    P(1), sums
    O += V(1) P(1)                               matrix core alone

The vector instructions of a half lie between the products of the other half, so that a wave by itself keeps both units busy for half
of its time; the other wave of the SIMD, of another workgroup and at another place of its tile, fills the rest.  Operands come from LDS
with DEPTH of them in flight, each waited for by count (6 take eight registers more, which
the code around the loop is short of: prompt pieces 456 us, 443 with 4, 443 with 3).  The next tile's loads are issued between the products of S(0).  The wave's priority
follows the phases, so that the two waves of a SIMD move apart and stay apart: the one nearest the end of its vector work goes first, the one in
the last phase, which only the matrix core holds up, goes last.  1280x720 chunk, priorities by phase: all equal 2550 us, 1 1 1 0 2455, 0 0 1 0 2348,
1 1 2 0 2295; 1 0 0 1 2570.  Before the products of a half its sums are looked at: where one is over
32768, or is no number, the statement ends, O as it was before that half, and the caller takes the rest of the tile another way.

Why asm: written in C++ the compiler read most operands right before their use (a wait of 64 to 128 cycles each), and took 250 vector
and 100 scalar instructions a tile besides the products where 112 and 45 do.  1280x720 chunk and twelve cached frames: 3509 us in
C++, 2990 us here (before its workgroups shared tiles in L2).

The statement carries its own waits and wait states (the compiler's hazard recogniser does not look into asm):
  * a vector instruction keeps 8 wait states from a product whose result it reads: at least nine instructions lie between the last
    product of S(h) and the first instruction that reads it, and the statement ends with two s_nop 7;
  * a product keeps 2 from a vector instruction that writes an operand of it: the sums are looked at in between;
  * an accumulator is reused four products later at the earliest;
  * no instruction uses the result of an exponential issued right before it;
  * one instruction lies between a write of m0 and the load into LDS that uses it.

Run this script after changing Layout in df_paged_attn.hip or the schedule; the include is committed and tests/test_paged_tiles.py
checks that it is what this script writes.
"""
import os

KT = 64
DEPTH = 4
STAGE = 256 - 4 * DEPTH
P = {(h, qb): STAGE - 16 + 8 * h + 4 * qb for h in range(2) for qb in range(2)}
S = {(kb, qb): STAGE - 48 + 8 * kb + 4 * qb for kb in range(4) for qb in range(2)}
Q0 = STAGE - 80
Q = {(ks, qb): Q0 + 8 * ks + 4 * qb for ks in range(4) for qb in range(2)}
O0 = Q0 - 64
O = {(db, qb): O0 + 8 * db + 4 * qb for db in range(8) for qb in range(2)}
TMP = O0 - 12                                    # three groups of four exponentials
PRIORITY = (1, 1, 2, 0)                          # of the wave, by phase
DK, DV = 64, 68                                  # descriptors


def quad(r):
    return f"v[{r}:{r + 3}]"


def half_softmax(h, pack):
    """P(h) and its sums in four groups of four values, three groups in flight."""
    groups = [(2 * h + u, qb) for u in range(2) for qb in range(2)]
    tmp = lambda i: TMP + 4 * (i % 3)
    out = []
    for i in range(len(groups) + 2):
        if i < len(groups):
            kb, qb = groups[i]
            out += [f"v_fma_f32 v{tmp(i) + v}, v{S[kb, qb] + v}, %[c], %[nm{qb}]" for v in range(4)]
        if 1 <= i <= len(groups):
            out += [f"v_exp_f32 v{tmp(i - 1) + v}, v{tmp(i - 1) + v}" for v in range(4)]
        if i >= 2:
            kb, qb = groups[i - 2]
            e = [f"v{tmp(i - 2) + v}" for v in range(4)]
            p = P[h, qb] + 2 * (kb % 2)
            if kb % 2 == 0:
                out += [f"v_add_f32 %[a{qb}], {e[0]}, {e[1]}", f"v_add_f32 %[b{qb}], {e[2]}, {e[3]}"]
            else:
                out += [f"v_add_f32 %[{'ab'[v // 2]}{qb}], %[{'ab'[v // 2]}{qb}], {e[v]}" for v in (0, 2, 1, 3)]
            out += [f"{pack} v{p + v}, {e[2 * v]}, {e[2 * v + 1]}" for v in range(2)]
    return out + [f"v_add_f32 %[a{qb}], %[a{qb}], %[b{qb}]" for qb in range(2)]


def look(h, buf):
    """Ends the statement where the weights of half h are too large, else takes its sums."""
    return ["v_add_f32 %[b0], %[a0], %[a1]",
            "v_cmp_nge_f32 vcc, %[most], %[b0]",
            f"s_cbranch_vccnz .Ldf_over{h}_%=",
            "v_add_f32 %[l0], %[l0], %[a0]",
            "v_add_f32 %[l1], %[l1], %[a1]"]


def tile(D, mfma, pack, buf):
    rowb, tile_bytes = 2 * D, KT * 2 * D
    at = buf * 2 * tile_bytes
    ops = []                                     # (phase, reads, products)
    for h in range(2):
        for ks in range(D // 32):
            for kb in (2 * h, 2 * h + 1):
                off = at + (32 * h + 4 * (kb % 2)) * rowb
                ops.append((h, [f"ds_read_b128 @, %[k{ks}] offset:{off}"],
                            [f"{mfma} {quad(S[kb, qb])}, @, {quad(Q[ks, qb])}, {quad(S[kb, qb]) if ks else 0}" for qb in range(2)]))
    for h in range(2):
        for db in range(D // 16):
            ops.append((2 + h, [f"ds_read_b64_tr_b16 @, %[v{db}] offset:{at + (32 * h + 4 * u) * rowb}" for u in range(2)],
                        [f"{mfma} {quad(O[db, qb])}, @, {quad(P[h, qb])}, {quad(O[db, qb])}" for qb in range(2)]))
    slot = lambda i: STAGE + 4 * (i % DEPTH)
    lines = []

    def issue(i):
        if i < len(ops):
            w = 4 // len(ops[i][1])
            for k, r in enumerate(ops[i][1]):
                lines.append(r.replace("@", f"v[{slot(i) + w * k}:{slot(i) + w * k + w - 1}]"))

    beside = {0: bring(D, buf), 1: half_softmax(0, pack), 2: half_softmax(1, pack)}
    for i in range(DEPTH):
        issue(i)
    for phase in range(4):
        mine = [i for i, o in enumerate(ops) if o[0] == phase]
        lines.append(f"s_setprio {PRIORITY[phase]}")
        vector = list(beside.get(phase, []))
        # the first vector instruction of a phase reads what the last products of the phase before have written
        skip = 3 if phase == 1 else 0
        products = 2 * (len(mine) - skip)
        done = 0
        for j, i in enumerate(mine):
            pending = sum(len(o[1]) for o in ops[i + 1:i + DEPTH])
            lines.append(f"s_waitcnt lgkmcnt({pending})")
            for k, m in enumerate(ops[i][2]):
                lines.append(m.replace("@", quad(slot(i))))
                if k:
                    issue(i + DEPTH)
                if j >= skip and vector:
                    part = 2 * (j - skip) + k + 1
                    upto = (len(vector) * part + products - 1) // products
                    lines += vector[done:upto]
                    done = upto
        lines += vector[done:]
        if phase in (1, 2):
            lines += look(phase - 1, buf)
    return lines


def bring(D, buf):
    """The next tile's rows of the wave into the other buffer."""
    rowb, tile_bytes, loads = 2 * D, KT * 2 * D, D // 32
    to = (buf ^ 1) * 2 * tile_bytes
    lines = ["v_readlane_b32 %[x], %[slots], %[i]",
             "s_add_i32 %[i], %[i], 1",
             "s_mul_hi_u32 %[y], %[x], %[stride]",
             "s_mul_i32 %[x], %[x], %[stride]",
             f"s_add_u32 s{DK}, %[klo], %[x]",
             f"s_addc_u32 s{DK + 1}, %[khi], %[y]",
             f"s_add_u32 s{DV}, %[vlo], %[x]",
             f"s_addc_u32 s{DV + 1}, %[vhi], %[y]"]
    for which, d in (("k", DK), ("v", DV)):
        for n in range(loads):
            off = to + (tile_bytes if which == "v" else 0) + 1024 * n
            lines += [f"s_add_u32 m0, %[to], {off:#x}", "s_nop 0", f"buffer_load_dwordx4 %[{which}o{n}], s[{d}:{d + 3}], 0 offen lds"]
    return lines


def statement(D, fp16):
    mfma = "v_mfma_f32_16x16x32_f16" if fp16 else "v_mfma_f32_16x16x32_bf16"
    pack = "v_cvt_pk_f16_f32" if fp16 else "v_cvt_pk_bf16_f32"
    lines = [f"s_mov_b32 s{DK + 2}, %[bytes]", f"s_mov_b32 s{DK + 3}, 0x20000", f"s_mov_b32 s{DV + 2}, %[bytes]", f"s_mov_b32 s{DV + 3}, 0x20000",
             "s_mov_b32 %[due], 0",
             "s_cmp_eq_u32 %[buf], 0", "s_cbranch_scc0 .Ldf_b1_%="]
    for buf in range(2):
        lines.append(f".Ldf_b{buf}_%=:")
        lines += ["s_waitcnt vmcnt(0)", "s_barrier"]
        lines += tile(D, mfma, pack, buf)
        lines += ["s_sub_i32 %[n], %[n], 1", "s_cmp_eq_u32 %[n], 0"]
        lines += ["s_cbranch_scc1 .Ldf_end_%="] if buf == 0 else ["s_cbranch_scc0 .Ldf_b0_%=", "s_branch .Ldf_end_%="]
    lines += [".Ldf_over1_%=:", "s_mov_b32 %[due], 1", ".Ldf_over0_%=:", "s_add_i32 %[due], %[due], 1", "s_waitcnt lgkmcnt(0)",
              ".Ldf_end_%=:", "s_setprio 0", "s_nop 7", "s_nop 7"]
    KS, DB, loads = D // 32, D // 16, D // 32
    outs = [f'"+{{{quad(O[db, qb])}}}"(o[{db}][{qb}])' for db in range(DB) for qb in range(2)]
    outs += [f'[l{qb}] "+v"(l[{qb}])' for qb in range(2)]
    outs += ['[i] "+s"(i)', '[n] "+s"(n)', '[due] "=&s"(due)', '[x] "=&s"(x)', '[y] "=&s"(y)']
    outs += [f'[{a}{qb}] "=&v"({a}_[{qb}])' for a in "ab" for qb in range(2)]
    outs += [f'"=&{{s[{d}:{d + 3}]}}"({v})' for d, v in ((DK, "dk"), (DV, "dv"))]
    ins = [f'"{{{quad(Q[ks, qb])}}}"(q[{ks}][{qb}])' for ks in range(KS) for qb in range(2)]
    ins += [f'[nm{qb}] "v"(nm[{qb}])' for qb in range(2)]
    ins += [f'[k{ks}] "v"(a.k[{ks}])' for ks in range(KS)] + [f'[v{db}] "v"(a.v[{db}])' for db in range(DB)]
    ins += [f'[{w}o{n}] "v"(a.{w}o[{n}])' for w in "kv" for n in range(loads)]
    ins += ['[slots] "v"(a.slots)'] + [f'[{n}] "s"(a.{n})' for n in ("klo", "khi", "vlo", "vhi", "stride", "bytes", "to", "buf", "c", "most")]
    clob = ['"vcc"', '"scc"', '"memory"'] + [f'"v{r}"' for r in list(range(TMP, TMP + 12)) + list(range(S[0, 0], 256))]
    body = "\n".join(f'      "{x}\\n\\t"' for x in lines)
    T = "Fp16" if fp16 else "Bf16"
    return f"""template <>
__device__ __forceinline__ int seen_tiles<{T}, {D}>(const SeenTiles<{D}> &a, const s16x8 (&q)[{KS}][2], f32x4 (&o)[{DB}][2], float (&l)[2],
                                                    const float (&nm)[2], int &i, int n) {{
  static_assert(Layout<{D}>::ROWB == {2 * D} && Layout<{D}>::LPG == {loads} && kManyKeys == {KT}, "run gen_paged_tiles.py");
  int due, x, y;
  float a_[2], b_[2];
  u32x4 dk, dv;
  asm volatile(
{body}
      : {', '.join(outs)}
      : {', '.join(ins)}
      : {', '.join(clob)});
  return due;
}}
"""


def operands(lines, ops, depth):
    """The operands' reads, `depth` of them ahead, and the products of each behind the wait for it."""
    slot = lambda i: STAGE + 4 * (i % DEPTH)

    def issue(i):
        if i < len(ops):
            w = 4 // len(ops[i][0])
            for k, r in enumerate(ops[i][0]):
                lines.append(r.replace("@", f"v[{slot(i) + w * k}:{slot(i) + w * k + w - 1}]"))

    for i in range(depth):
        issue(i)
    for i, (_, products) in enumerate(ops):
        lines.append(f"s_waitcnt lgkmcnt({sum(len(o[0]) for o in ops[i + 1:i + depth])})")
        lines += [m.replace("@", quad(slot(i))) for m in products]
        issue(i + depth)
    return lines + ["s_nop 7", "s_nop 7"]


def one_product(D, fp16, second):
    """S^T = K Q^T or O^T += V^T P^T of a whole tile by itself, for tiles with something between the two."""
    rowb, KS, DB = 2 * D, D // 32, D // 16
    mfma = "v_mfma_f32_16x16x32_f16" if fp16 else "v_mfma_f32_16x16x32_bf16"
    T = "Fp16" if fp16 else "Bf16"
    if second:
        ops = [([f"ds_read_b64_tr_b16 @, %[v{db}] offset:{(32 * h + 4 * u) * rowb}" for u in range(2)],
                [f"{mfma} {quad(O[db, qb])}, @, {quad(P[h, qb])}, {quad(O[db, qb])}" for qb in range(2)])
               for h in range(2) for db in range(DB)]
        outs = [f'"+{{{quad(O[db, qb])}}}"(o[{db}][{qb}])' for db in range(DB) for qb in range(2)]
        ins = [f'"{{{quad(P[h, qb])}}}"(w[{h}][{qb}])' for h in range(2) for qb in range(2)]
        ins += [f'[v{db}] "v"(first ^ {32 * db}u)' for db in range(DB)]
        head = f"void values_of<{T}, {D}>(unsigned first, const s16x8 (&w)[2][2], f32x4 (&o)[{DB}][2])"
        lines = ["s_waitcnt lgkmcnt(0)", "s_nop 1"]
    else:
        ops = [([f"ds_read_b128 @, %[k{ks}] offset:{(32 * (kb // 2) + 4 * (kb % 2)) * rowb}"],
                [f"{mfma} {quad(S[kb, qb])}, @, {quad(Q[ks, qb])}, {quad(S[kb, qb]) if ks else 0}" for qb in range(2)])
               for ks in range(KS) for kb in range(4)]
        outs = [f'"=&{{{quad(S[kb, qb])}}}"(s[{kb}][{qb}])' for kb in range(4) for qb in range(2)]
        ins = [f'"{{{quad(Q[ks, qb])}}}"(q[{ks}][{qb}])' for ks in range(KS) for qb in range(2)]
        ins += [f'[k{ks}] "v"(first ^ {64 * ks}u)' for ks in range(KS)]
        head = f"void scores_of<{T}, {D}>(unsigned first, const s16x8 (&q)[{KS}][2], f32x4 (&s)[4][2])"
        lines = ["s_waitcnt lgkmcnt(0)"]
    body = "\n".join(f'      "{x}\\n\\t"' for x in operands(lines, ops, DEPTH))
    clob = ['"memory"'] + [f'"v{r}"' for r in range(STAGE, 256)]
    return f"""template <>
__device__ __forceinline__ {head} {{
  asm volatile(
{body}
      : {', '.join(outs)}
      : {', '.join(ins)}
      : {', '.join(clob)});
}}
"""


def text():
    head = "// Generated by gen_paged_tiles.py - do not edit; see that script for the schedule and its reasons.\n"
    every = [(D, fp16) for D in (128, 64) for fp16 in (False, True)]
    return head + "\n".join([statement(*x) for x in every] + [one_product(*x, second) for x in every for second in (False, True)])


OUT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "df_paged_tiles.inc")

if __name__ == "__main__":
    with open(OUT, "w") as f:
        f.write(text())
    print("wrote", OUT)
