"""The paged operators on the CPU: layout of the argument structs, what the library refuses before it touches the GPU, and what the
binding refuses because the library could not see it (types, shapes, places)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from tests import paged_util as pu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    if not os.path.exists(os.path.join(ROOT, "paper_2601_20499_amd", "libdf_hip.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2601_20499_amd import binding
    return binding


def test_struct_layout_matches_c(b, tmp_path):
    structs = [b.df_paged_cache, b.df_page_map_args, b.df_paged_append_args, b.df_paged_attn_args]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "df.h"', 'int main(void){']
    for st in structs:
        lines.append(f'printf("{st.__name__} %zu\\n", sizeof({st.__name__}));')
        lines += [f'printf("{st.__name__}.{f} %zu\\n", offsetof({st.__name__}, {f}));' for f, _ in st._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    got = dict(zip(out[0::2], map(int, out[1::2])))
    for st in structs:
        assert got[st.__name__] == C.sizeof(st)
        for f, _ in st._fields_:
            assert got[f"{st.__name__}.{f}"] == getattr(st, f).offset, (st.__name__, f)


def _cache(b, **kw):
    """A valid cache of made-up addresses, which nothing reads: every call below is refused on the host."""
    c = b.df_paged_cache()
    for f in ("k_pages", "v_pages", "block_table", "len", "sink_cap", "win_cap", "free_pages", "n_free"):
        setattr(c, f, 0x10000)
    c.cap_stride, c.B, c.H_kv, c.d, c.dtype, c.n_pages, c.page_tokens, c.max_pages = 4, 3, 4, 128, b.DF_BF16, 100, 16, 8
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _calls(b, cache, **kw):
    """The three calls on a cache, each with the fields of `kw` that it has."""
    m, p, a = b.df_page_map_args(), b.df_paged_append_args(), b.df_paged_attn_args()
    for x in (m, p, a):
        x.cache = C.pointer(cache)
        x.total_new = 10
    m.cu_new = m.slot_map = m.len_out = m.n_free_out = m.status = 0x20000
    p.k_new = p.v_new = p.slot_map = 0x20000
    p.stride_tok, p.stride_head = 512, 128
    a.q = a.k_cur = a.v_cur = a.cu_new = a.out = 0x20000
    a.q_stride_tok = a.o_stride_tok = 1024
    a.kc_stride_tok, a.q_stride_head, a.o_stride_head, a.kc_stride_head = 512, 128, 128, 128
    a.H_q, a.max_new, a.block, a.softmax_scale, a.workspace, a.workspace_bytes = 8, 4, 1, 0.1, 0x100000, 1 << 30
    for x in (m, p, a):
        for k, v in kw.items():
            if k in dict(x._fields_):
                setattr(x, k, v)
    return (lambda: b.lib.df_page_map(C.byref(m), None), lambda: b.lib.df_paged_append(C.byref(p), None),
            lambda: b.lib.df_paged_attn(C.byref(a), None))


@pytest.mark.parametrize("field,value,code", [
    ("B", 0, 2), ("B", -1, 2), ("B", (1 << 16) + 1, 6), ("H_kv", 0, 2), ("H_kv", 65, 3), ("d", 96, 3), ("d", 0, 3), ("dtype", 2, 3), ("dtype", -1, 3),
    ("n_pages", 0, 2), ("n_pages", (1 << 30) + 1, 6), ("page_tokens", 0, 2), ("page_tokens", 8, 3), ("page_tokens", 48, 3),
    ("page_tokens", 2048, 3), ("max_pages", 0, 2), ("max_pages", (1 << 30) + 1, 6), ("k_pages", None, 1), ("v_pages", None, 1), ("block_table", None, 1),
    ("len", None, 1), ("sink_cap", None, 1), ("win_cap", None, 1), ("k_pages", 0x10008, 4), ("v_pages", 0x10002, 4), ("cap_stride", 3, 2)])
def test_every_call_refuses_a_bad_cache(b, field, value, code):
    for call in _calls(b, _cache(b, **{field: value})):
        assert call() == code, field
    for call in (b.lib.df_page_map, b.lib.df_paged_append, b.lib.df_paged_attn):
        assert call(None, None) == b.DF_ERR_NULL


@pytest.mark.parametrize("which,kw,code", [
    (0, dict(total_new=-1), 2), (0, dict(total_new=(1 << 30) + 1), 6), (0, dict(cu_new=None), 1), (0, dict(slot_map=None), 1),
    (0, dict(len_out=None), 1), (0, dict(n_free_out=None), 1), (0, dict(status=None), 1),
    (1, dict(total_new=-1), 2), (1, dict(k_new=None), 1), (1, dict(v_new=None), 1), (1, dict(slot_map=None), 1), (1, dict(k_new=0x20008), 4),
    (1, dict(stride_tok=12), 4), (1, dict(stride_tok=0), 4), (1, dict(stride_head=-8), 4),
    (2, dict(q=None), 1), (2, dict(out=None), 1), (2, dict(cu_new=None), 1), (2, dict(k_cur=None), 1), (2, dict(v_cur=None), 1),
    (2, dict(H_q=0), 2), (2, dict(H_q=6), 2), (2, dict(H_q=4 * 65), 3), (2, dict(total_new=0), 2), (2, dict(max_new=0), 2), (2, dict(max_new=11), 2),
    (2, dict(block=0), 2), (2, dict(softmax_scale=0.0), 6), (2, dict(softmax_scale=-1.0), 6), (2, dict(softmax_scale=float("nan")), 6),
    (2, dict(softmax_scale=float("inf")), 6), (2, dict(q=0x20004), 4), (2, dict(out=0x20004), 4), (2, dict(k_cur=0x20004), 4),
    (2, dict(q_stride_tok=4), 4), (2, dict(o_stride_head=4), 4), (2, dict(kc_stride_tok=-8), 4), (2, dict(kc_stride_tok=(1 << 26) + 8), 6),
    (2, dict(workspace=None), 5), (2, dict(workspace_bytes=1000), 5), (2, dict(workspace=0x100010), 4),
    (2, dict(total_new=1 << 30, max_new=1 << 30), 6)])
def test_refusals(b, which, kw, code):
    assert _calls(b, _cache(b), **kw)[which]() == code


def test_calls_without_tokens_do_nothing(b):
    assert _calls(b, _cache(b), total_new=0)[1]() == b.DF_OK
    for f in ("free_pages", "n_free"):                       # only the map needs them
        calls = _calls(b, _cache(b, **{f: None}), workspace=None)
        assert calls[0]() == b.DF_ERR_NULL and calls[2]() == b.DF_ERR_WORKSPACE


def test_workspace_sizes(b):
    for hq, hkv, d, n in ((0, 1, 128, 1), (3, 2, 128, 1), (1, 0, 128, 1), (65, 65, 128, 1), (1, 1, 80, 1), (1, 1, 64, 0), (2, 1, 64, 1 << 30)):
        assert b.df_paged_workspace_bytes(hq, hkv, d, n) == 0
    few, many = b.df_paged_workspace_bytes(32, 8, 128, 1), b.df_paged_workspace_bytes(32, 8, 128, 4096)
    assert 0 < few < many <= 80 << 20
    assert b.df_paged_workspace_bytes(64, 1, 64, 1 << 20) > 0


# ---- the binding ----------------------------------------------------------------------------------------------------------------

def _batch(**kw):
    return pu.Batch(0, [20, 5], [3, 4], [(0, pu.FULL), (4, 16)], G=2, d=64, device="cpu", **kw)


@pytest.mark.parametrize("spoil", ["dtype", "pages", "table", "length", "caps", "free", "n_free", "strided"])
def test_cache_refuses_what_the_library_cannot_see(b, spoil):
    x = _batch()
    if spoil == "dtype":
        x.k_pages = x.k_pages.float()
    if spoil == "pages":
        x.v_pages = x.v_pages[:-1].contiguous()
    if spoil == "table":
        x.table = x.table.long()
    if spoil == "length":
        x.length = x.length[:1]
    if spoil == "caps":
        x.win = x.win[:1]
    if spoil == "free":
        x.free = x.free[:-1]
    if spoil == "n_free":
        x.n_free = x.n_free.long()
    if spoil == "strided":
        x.table = torch.cat([x.table, x.table], 2)[:, :, :x.max_pages]
    with pytest.raises(ValueError):
        x.cache(b)


def test_calls_refuse_what_the_library_cannot_see(b):
    x = _batch()
    c = x.cache(b)
    out, ws = torch.empty_like(x.q), torch.empty(1 << 20, dtype=torch.uint8)
    slots, status = torch.zeros(7, 2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32)
    good = dict(q=x.q, k_cur=x.k_new, v_cur=x.v_new, cache=c, cu_new=x.cu, out=out, softmax_scale=1.0, workspace=ws)
    other = lambda t: t.to(torch.float16)
    for bad in (dict(q=other(x.q)), dict(out=other(out)), dict(out=out[:-1]), dict(k_cur=x.k_new[:-1], v_cur=x.v_new[:-1]), dict(k_cur=None),
                dict(v_cur=x.v_new.transpose(0, 1).contiguous().transpose(0, 1)), dict(cu_new=x.cu.long()), dict(cu_new=x.cu[:-1]),
                dict(lse_out=torch.empty(7, 4)), dict(q=x.q.transpose(1, 2)), dict(k_cur=x.k_new[:, :1], v_cur=x.v_new[:, :1])):
        with pytest.raises(ValueError):
            b.df_paged_attn(**{**good, **bad})
    for bad in (dict(slot_map=slots.int()), dict(slot_map=slots[:, :1]), dict(status=status.long()), dict(release=status),
                dict(len_out=status), dict(n_free_out=x.length), dict(cu_new=x.cu[1:])):
        with pytest.raises(ValueError):
            b.df_page_map(**{**dict(cache=c, cu_new=x.cu, slot_map=slots, status=status), **bad})
    for bad in (dict(k_new=other(x.k_new)), dict(v_new=x.v_new[:-1]), dict(slot_map=slots[:-1]), dict(slot_map=slots.int())):
        with pytest.raises(ValueError):
            b.df_paged_append(**{**dict(cache=c, k_new=x.k_new, v_new=x.v_new, slot_map=slots), **bad})
    with pytest.raises(b.DfError) as e:                       # and what it can see comes back as its status
        b.df_paged_attn(**{**good, "workspace": None}, stream=0)
    assert e.value.status == b.DF_ERR_WORKSPACE


# ---- the model itself -------------------------------------------------------------------------------------------------------------

def test_model_keeps_what_a_list_of_tokens_keeps():
    """Slots, seen from the other side: after any steps a head's filled slots hold its first tokens and its last ones."""
    rng = np.random.default_rng(3)
    for s, w in ((0, 0), (5, 0), (0, 7), (3, 11), (2, pu.FULL), (40, 1)):
        m = pu.Model(1, [[(s, w)]], 100, 16, 100)
        held, n = {}, 0
        for _ in range(12):
            new = int(rng.integers(0, 20))
            for i, row in enumerate(m.map([new])):
                if row[0] >= 0:
                    held[row[0]] = n + i
            n += new
            assert sorted(held.values()) == pu.held_positions(n, s, w)


def test_model_attention_is_softmax_over_what_is_seen():
    x = pu.Batch(4, [9], [3], [(2, 4)], d=64, device="cpu")
    out, _, lse, keys, _ = x.reference(2)
    assert keys.tolist() == [[2 + 4 + 2, 2 + 4 + 2, 2 + 2 + 3]]    # the last token's block begins at 2: it sees two tokens less behind it
    back, ahead = [0, 1, 7, 8], [0, 1, 2]
    k = torch.cat([x.hist[0][0][0][back], x.k_new[ahead, 0]]).double()
    v = torch.cat([x.hist[0][0][1][back], x.v_new[ahead, 0]]).double()
    s = (k @ x.q[2, 0].double()) * x.scale
    assert np.allclose(out[2, 0], (torch.softmax(s, 0) @ v).numpy(), atol=1e-12)
    assert np.isclose(lse[0, 2], torch.logsumexp(s, 0).item(), atol=1e-12)
