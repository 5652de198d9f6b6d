"""Paged KV cache without a GPU: the index arithmetic of its kernels (compiled for the host) against Eqs. 1 and 3 row by row,
and what the calls refuse."""
import ctypes
import dataclasses
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2604_24432_b200 import binding as ksa
from paper_2604_24432_b200 import build as ksa_build
from tests import paged_ref as ref

HOST = r"""
#include "ksa_paged_index.h"
struct Given { int kk, m, C, rows, num_pages; unsigned flags; };
struct Shape : Given {
    ksa::PagedDiv by_chunk, by_k, by_m;
    Shape(const Given& g) : Given(g), by_chunk(ksa::PagedDiv::by(g.kk + g.m)), by_k(ksa::PagedDiv::by(g.kk)), by_m(ksa::PagedDiv::by(g.m)) {}
};
extern "C" {
int divide(int x, int d) { return ksa::PagedDiv::by(d)(x); }
int place(const Given* g, int row, int* summ) { Shape shape(*g); const Shape* a = &shape; bool s; int x = ksa::paged_place(*a, row, s); *summ = s; return x; }
int texts(const Given* g, int row) { Shape shape(*g); const Shape* a = &shape; return ksa::paged_texts(*a, row); }
int entry(const Given* g, int e) { Shape shape(*g); const Shape* a = &shape; return ksa::paged_entry(*a, e); }
int lengths_ok(const Given* g, int row0, int r1, int first) { Shape shape(*g); const Shape* a = &shape; return ksa::paged_lengths_ok(*a, row0, r1, first); }
void view(const Given* g, int summ, int x, int* v) { Shape shape(*g); const Shape* a = &shape; auto w = ksa::paged_view(*a, summ, x); v[0] = w.t_lo; v[1] = w.t_hi; v[2] = w.s_lo; v[3] = w.s_hi; }
void tile_view(const Given* g, int summ, int x0, int n, int* v) { Shape shape(*g); const Shape* a = &shape; ksa::PagedTile t{0, summ != 0, false, x0, n, 0, 0}; auto w = ksa::paged_tile_view(*a, t); v[0] = w.t_lo; v[1] = w.t_hi; v[2] = w.s_lo; v[3] = w.s_hi; }
void range(const Given* g, int first, int n, int summ, int* v) { Shape shape(*g); const Shape* a = &shape; auto r = ksa::paged_range(*a, first, n, summ != 0); v[0] = r.lo; v[1] = r.hi; v[2] = r.gap_lo; v[3] = r.gap_hi; }
int token(const Given* g, int first, int i, int* summ) { Shape shape(*g); const Shape* a = &shape; ksa::PagedTile t{0, false, true, first, 0, 0, first}; bool s; int x = ksa::paged_token(*a, t, i, s); *summ = s; return x; }
// tiles of 16 rows: (stream, first row, first row seen of 16 as bits, all seen) of each
int walk(const Given* g, int mixed, int summ, int x0, int n, int split, int parts, int* out) { Shape shape(*g); const Shape* a = &shape;
    ksa::PagedTile t{0, summ != 0, mixed != 0, x0, n, 0, x0};
    ksa::PagedWalk<16> w;
    w.init(*a, t, split, parts);
    for (int j = w.j0; j < w.j1; ++j, out += 5) {
        auto k = w.at(j);
        out[0] = k.summ; out[1] = k.x0; out[2] = 0; out[3] = k.sees_all(); out[4] = 0;
        for (int i = 0; i < 16; ++i) { out[2] |= k.sees(k.x0 + i) << i; if (i % 4 == 0) out[4] |= k.sees_any(k.x0 + i, 4) << (i / 4); }
    }
    return w.j1 - w.j0;
}
long long row(const Given* g, int summ, int x, int row0, int first) { Shape shape(*g); const Shape* a = &shape; ksa::PagedTile t{0, summ != 0, false, 0, 0, row0, first}; return ksa::paged_row(*a, t, x); }
}
"""


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("kk", "m", "C", "rows", "num_pages")] + [("flags", ctypes.c_uint)]


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    src, so = d / "index.cpp", d / "index.so"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", ksa_build.CSRC, str(src), "-o", str(so)], check=True)
    L = ctypes.CDLL(str(so))
    L.row.restype = ctypes.c_longlong
    return L


@pytest.mark.parametrize("k,m,C,flags", [(8, 1, 3, 0), (8, 1, 0, 0), (64, 8, 1, 0), (1, 1, 5, 0), (3, 2, 2, 1), (8, 0, 1 << 20, 0), (4, 0, 2, 0), (200, 3, 1, 1)])
def test_rows_places_and_views(index, k, m, C, flags):
    a = Shape(k, m, C, 1 << 20, 10, flags)
    rows = 4 * (k + m) * max(1, min(C, 4)) + 5
    where = ref.places(k, m, rows)
    out4 = (ctypes.c_int * 4)()
    for row, (is_summ, x) in enumerate(where):
        s = ctypes.c_int()
        assert (index.place(ctypes.byref(a), row, ctypes.byref(s)), bool(s.value)) == (x, is_summ)
        assert index.texts(ctypes.byref(a), row) == sum(not w[0] for w in where[:row])
        assert index.row(ctypes.byref(a), int(is_summ), x, 70, 3) == 70 + row - 3
        index.view(ctypes.byref(a), int(is_summ), x, out4)
        see = ref.visible(k, m, C, row, rows, bool(flags & 1))
        text = [w[1] for i, w in enumerate(where) if see[i] and not w[0]]
        summ = [w[1] for i, w in enumerate(where) if see[i] and w[0]]
        assert list(range(out4[0], out4[1])) == text and list(range(out4[2], max(out4[2], out4[3]))) == summ, row
    # a tile's view covers what its rows see, and is no wider than from its first to its last
    for kind in (False, True):
        have = [i for i, w in enumerate(where) if w[0] == kind]
        for lo in range(0, len(have), max(1, len(have) // 7)):
            for n in (1, 5, 16):
                part = have[lo:lo + n]
                if not part:
                    continue
                index.tile_view(ctypes.byref(a), int(kind), where[part[0]][1], len(part), out4)
                see = np.any([ref.visible(k, m, C, i, rows, bool(flags & 1)) for i in part], axis=0)
                text = [w[1] for i, w in enumerate(where) if see[i] and not w[0]]
                summ = [w[1] for i, w in enumerate(where) if see[i] and w[0]]
                assert (min(text), max(text) + 1) == (out4[0], out4[1])
                assert (summ == [] and out4[2] >= out4[3]) or (min(summ), max(summ) + 1) == (out4[2], out4[3])


@pytest.mark.parametrize("k,m,C,flags", [(8, 1, 3, 0), (8, 1, 0, 0), (64, 8, 1, 0), (1, 1, 5, 0), (3, 2, 2, 1), (8, 0, 1 << 20, 0), (4, 0, 2, 0), (5, 3, 1, 0)])
def test_what_a_run_of_rows_sees(index, k, m, C, flags):
    a = Shape(k, m, C, 1 << 20, 10, flags)
    rows = 5 * (k + m) * max(1, min(C, 3)) + 4
    where = ref.places(k, m, rows)
    sees = [ref.visible(k, m, C, i, rows, bool(flags & 1)) for i in range(rows)]
    out4 = (ctypes.c_int * 4)()
    for first in range(0, rows, max(1, rows // 60)):
        for n in (1, 2, k, k + m, 3 * (k + m) + 1):
            if first + n > rows:
                continue
            see = np.any(sees[first:first + n], axis=0)
            for kind in (False, True):
                index.range(ctypes.byref(a), first, n, int(kind), out4)
                got = [x for x in range(out4[0], out4[1]) if not out4[2] <= x < out4[3]]
                want = [w[1] for i, w in enumerate(where) if see[i] and w[0] == kind]
                # (text between the windows of two rows that are far apart is no case: a run's windows overlap or touch)
                assert got == want, (first, n, kind)


@pytest.mark.parametrize("k,m,C,flags", [(8, 1, 3, 0), (8, 1, 0, 0), (64, 8, 1, 0), (1, 1, 5, 0), (3, 2, 2, 1), (8, 0, 1 << 20, 0), (2, 1, 40, 0), (5, 3, 1, 0)])
def test_key_tiles_of_a_query_tile(index, k, m, C, flags):
    """Every key tile once, over any number of parts; of it exactly the rows that some row of the query tile sees."""
    a = Shape(k, m, C, 1 << 20, 10, flags)
    rows = 3 * (k + m) * max(2, min(C, 45)) + 4
    where = ref.places(k, m, rows)
    sees = [ref.visible(k, m, C, i, rows, bool(flags & 1)) for i in range(rows)]
    buf = (ctypes.c_int * (5 * 4096))()
    tiles = [(True, False, first, n, list(range(first, min(rows, first + n)))) for first in range(0, rows, max(1, rows // 40)) for n in (1, 2, 7, k + m, 40)]
    for kind in (False, True):
        of = [i for i, w in enumerate(where) if w[0] == kind]
        tiles += [(False, kind, where[of[lo]][1], len(of[lo:lo + n]), of[lo:lo + n]) for lo in range(0, len(of), max(1, len(of) // 30)) for n in (1, 5, 33)]
    for mixed, kind, x0, n, members in tiles:
        if mixed and len(members) < n:
            continue
        see = np.any([sees[i] for i in members], axis=0)
        want = {(w[0], w[1]) for i, w in enumerate(where) if see[i]}
        for parts in (1, 3):
            got, seen = [], set()
            for split in range(parts):
                cnt = index.walk(ctypes.byref(a), int(mixed), int(kind), x0, n, split, parts, buf)
                for j in range(cnt):
                    summ, first, bits, whole, quads = buf[5 * j:5 * j + 5]
                    got.append((bool(summ), first))
                    seen |= {(bool(summ), first + i) for i in range(16) if bits >> i & 1}
                    assert bool(whole) == (bits == 0xffff)
                    assert all(not (bits >> (4 * i) & 15) or quads >> i & 1 for i in range(4))     # (a run may be fetched for nothing, never missed)
            assert len(set(got)) == len(got) and all(f % 16 == 0 for _, f in got)
            assert seen == want, (mixed, kind, x0, n)
    s = ctypes.c_int()
    for i in range(30):
        assert (index.token(ctypes.byref(a), 11, i, ctypes.byref(s)), bool(s.value)) == (ref.places(k, m, 12 + i)[11 + i][1], ref.places(k, m, 12 + i)[11 + i][0])


def test_workspace_of_long_runs_over_e4m3():
    def need(**change):
        good = dict(struct_size=ctypes.sizeof(ksa.ksa_paged_params), batch=1, num_rows=1152, chunk_len=8, summaries_per_chunk=1, window_chunks=128,
                    num_q_heads=32, num_kv_heads=8, head_dim=128, softmax_scale=0.1, flags=0, kv_format=ksa.KSA_KV_E4M3, page_rows=64,
                    num_pages=7, text_cols=600, summ_cols=70, page_stride=65536, head_stride=8192, row_stride=128)
        n = ctypes.c_size_t()
        rc = ksa.lib().ksa_paged_workspace_bytes(ctypes.byref(ksa.ksa_paged_params(**{**good, **change})), ctypes.byref(n))
        return n.value if rc == 0 else rc
    pages = (130 * 8 + 1152) // 128 + 2 + 35
    assert need() == 2 * pages * 8 * 128 * 128 * 2 + (300 + 35) * 4
    assert need(num_rows=255) == need(batch=5) == need(kv_format=ksa.KSA_KV_BF16, page_stride=65536) == 0
    assert need(text_cols=5, num_rows=512) == 2 * (3 + 35) * 8 * 128 * 128 * 2 + (3 + 35) * 4
    assert need(window_chunks=1 << 30, chunk_len=8, summaries_per_chunk=0, summ_cols=0, text_cols=1 << 24) == 0       # over 2 GB: the cache itself
    assert need(head_dim=96) == ksa.KSA_ERR_UNSUPPORTED


def test_entries_and_lengths(index):
    a = Shape(8, 1, 3, 100, 10, 0)
    assert [index.entry(ctypes.byref(a), e) for e in (-1, 0, 9, 10, -2, 2**31 - 1, -2**31)] == [-1, 0, 9, -2, -2, -2, -2]
    ok = lambda *v: bool(index.lengths_ok(ctypes.byref(a), *v))
    assert ok(0, 0, 0) and ok(0, 100, 0) and ok(99, 100, 2**30 - 1) and ok(100, 100, 2**30)
    assert not ok(-1, 5, 0) and not ok(5, 4, 0) and not ok(0, 101, 0) and not ok(0, 1, -1) and not ok(0, 1, 2**30)
    assert not ok(-2**31, 2**31 - 1, 0) and not ok(0, -5, 0) and not ok(0, 1, 2**31 - 1)


def test_division(index):
    rng = np.random.default_rng(0)
    for d in [1, 2, 3, 5, 7, 8, 9, 64, 72, 127, 128, 641, 65535, 65536, 10**9, 2**30] + [int(x) for x in rng.integers(1, 2**31 - 1, 40)]:
        for x in [0, 1, d - 1, d, d + 1, 2 * d - 1, 2**31 - 1, 2**31 - 2, 2**30] + [int(v) for v in rng.integers(0, 2**31, 60)] + [int(q) * d + r for q in rng.integers(0, 2**31 // d + 1, 20) for r in (-1, 0)]:
            if 0 <= x < 2**31:
                assert index.divide(x, d) == x // d, (x, d)


def test_e4m3_reference_matches_torch():
    x = np.concatenate([np.linspace(-448, 448, 20001), ref.E4M3, (ref.E4M3[1:] + ref.E4M3[:-1]) / 2])
    x = torch.from_numpy(x).float().double().numpy()
    x[0] = 448.0
    codes, byte = ref.quantise_row(x)
    assert byte == 127
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (codes == want).all()


@pytest.fixture(scope="module", autouse=True)
def _built():
    ksa_build.build()


def _call(fn="append", kv_change=None, tensor_change=None, ws=None, **change):
    """Status of a call with made-up (never touched) pointers and no context: what is wrong is said before anything else."""
    D, Hkv, Hq, ps = change.get("head_dim", 128), 2, 8, 64
    good = dict(struct_size=ctypes.sizeof(ksa.ksa_paged_params), batch=2, num_rows=5, chunk_len=8, summaries_per_chunk=1, window_chunks=4,
                num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, softmax_scale=0.1, flags=0, kv_format=ksa.KSA_KV_E4M3, page_rows=ps,
                num_pages=7, text_cols=3, summ_cols=1, page_stride=Hkv * ps * D, head_stride=ps * D, row_stride=D,
                q_stride_tok=Hq * D, q_stride_head=D, k_stride_tok=Hkv * D, k_stride_head=D, v_stride_tok=Hkv * D, v_stride_head=D,
                o_stride_tok=Hq * D, o_stride_head=D)
    p = ksa.ksa_paged_params(**{**good, **change})
    kv = ksa.ksa_paged_kv(**{**{n: 0x10000 * (i + 1) for i, (n, _) in enumerate(ksa.ksa_paged_kv._fields_)}, **(kv_change or {})})
    x, y, z = {**dict(x=0x900000, y=0xA00000, z=0xB00000), **(tensor_change or {})}.values()
    L = ksa.lib()
    if fn == "attn":
        return L.ksa_paged_attn(None, ctypes.byref(kv), x, y, z, ws, 1 << 20, ctypes.byref(p), None)
    return getattr(L, "ksa_paged_" + fn)(None, ctypes.byref(kv), x, y, ctypes.byref(p), None)


BAD, UNSUP = ksa.KSA_ERR_INVALID_ARG, ksa.KSA_ERR_UNSUPPORTED


@pytest.mark.parametrize("fn", ["append", "gather", "attn"])
@pytest.mark.parametrize("change,want", [
    (dict(struct_size=8), BAD), (dict(batch=0), BAD), (dict(num_rows=-1), BAD), (dict(chunk_len=0), BAD), (dict(summaries_per_chunk=-1), BAD),
    (dict(window_chunks=-1), BAD), (dict(num_q_heads=7), BAD), (dict(num_kv_heads=0), BAD), (dict(head_dim=96), UNSUP),
    (dict(softmax_scale=0.0), BAD), (dict(softmax_scale=float("nan")), BAD), (dict(flags=2), BAD), (dict(flags=0x60), BAD), (dict(kv_format=2), BAD),
    (dict(page_rows=48), UNSUP), (dict(page_rows=256), UNSUP), (dict(page_rows=8), UNSUP), (dict(num_pages=0), BAD), (dict(text_cols=0), BAD),
    (dict(summ_cols=0), BAD), (dict(page_stride=-16), BAD), (dict(page_stride=0), BAD), (dict(head_stride=0), BAD), (dict(row_stride=1 << 38), UNSUP), (dict(row_stride=120), BAD), (dict(row_stride=64), BAD), (dict(head_stride=8), BAD),
    (dict(num_q_heads=130), UNSUP), (dict(num_rows=1 << 25), UNSUP), (dict(batch=70000), UNSUP), (dict(chunk_len=2**31 - 1), UNSUP),
    (dict(kv_change=dict(kpages=None)), BAD), (dict(kv_change=dict(vpages=0x10008)), BAD), (dict(kv_change=dict(kscale=None)), BAD),
    (dict(kv_change=dict(vscale=0x10004)), BAD), (dict(kv_change=dict(text_table=None)), BAD), (dict(kv_change=dict(summ_table=None)), BAD),
    (dict(kv_change=dict(cached=None)), BAD), (dict(kv_change=dict(cu_rows=None)), BAD), (dict(tensor_change=dict(x=None)), BAD),
    (dict(tensor_change=dict(y=0xA00008)), BAD), (dict(), BAD),        # all well but for the context
])
def test_refusals(fn, change, want):
    assert _call(fn, **change) == want


@pytest.mark.parametrize("fn,change", [("append", dict(k_stride_tok=12)), ("append", dict(v_stride_head=-8)), ("gather", dict(k_stride_tok=1 << 38)),
                                       ("attn", dict(q_stride_tok=4)), ("attn", dict(o_stride_head=-8)), ("attn", dict(tensor_change=dict(z=None))),
                                       ("attn", dict(tensor_change=dict(z=0xB00002))), ("attn", dict(ws=0xC00080))])
def test_refusals_of_row_tensors(fn, change):
    assert _call(fn, **change) == BAD


def test_null_structures():
    assert ksa.lib().ksa_paged_append(None, None, None, None, None, None) == BAD
    assert ksa.lib().ksa_paged_attn(None, None, None, None, None, None, 0, None, None) == BAD
    n = ctypes.c_size_t()
    assert ksa.lib().ksa_paged_workspace_bytes(None, ctypes.byref(n)) == BAD


def test_binding_refusals():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    good = dict(cached=i32(2), cu_rows=i32(3), text_table=i32(2, 4), summ_table=i32(2, 1))
    ksa.PagedBatch(**good)
    for bad in (dict(cu_rows=i32(2)), dict(cached=i32(2, 1)), dict(text_table=i32(3, 4)), dict(text_table=i32(8)), dict(cached=torch.zeros(2, dtype=torch.int64)),
                dict(summ_table=i32(4, 2).t()), dict(summ_table=i32(2, 4)[:, ::2])):
        with pytest.raises(ValueError):
            ksa.PagedBatch(**{**good, **bad})

    class Ctx:                                       # no device is needed to refuse
        device, handle = 0, None
    spec = ksa.PagedSpec(8, 1, 4, 8, 2, 128, 0.1, 64, 3, "bf16")
    pool = torch.zeros((3, 2, 64, 128), dtype=torch.bfloat16)
    for s, kw in ((dataclasses.replace(spec, fmt="int8"), {}), (spec, dict(kpages=pool)), (spec, dict(kpages=pool, vpages=pool)),
                  (spec, dict(kpages=pool, vpages=pool, kscale=pool, vscale=pool))):
        with pytest.raises(ValueError):
            ksa.PagedCache(Ctx, s, **kw)
