// Index arithmetic of the paged KV cache: which row is which token, where it lies, what it sees.  Plain C++ for both sides: the
// kernels use it, and the tests compile it for the host and compare it with Eqs. 1 and 3 row by row.
// `A` holds kk, m, C (chunk length, summaries, window), by_chunk, by_k, by_m (divisors k + m, k and m), flags, rows and num_pages.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define KSA_HD __host__ __device__ __forceinline__
#else
#define KSA_HD inline
#endif
#ifndef KSA_FLAG_SUMMARY_TEXT_ONLY
#define KSA_FLAG_SUMMARY_TEXT_ONLY 0x1u
#endif

namespace ksa {

// x / d for 0 <= x < 2^31 as a product: with l the least number with 2^l >= d and mul = floor(2^32 (2^l - d) / d) + 1,
// x / d = (floor(x mul / 2^32) + x) >> l (Granlund and Montgomery, 1994).  (A division is some twenty dependent instructions, and a kernel
// goes through about ten before its first load.)
struct PagedDiv {
    uint32_t mul; int32_t shift;
    static inline PagedDiv by(int d)                   // (host)
    {
        PagedDiv v{0, 0};
        if (d < 1) return v;
        while ((1ll << v.shift) < d) ++v.shift;
        v.mul = (uint32_t)((((1ull << v.shift) - (uint64_t)d) << 32) / (uint64_t)d + 1);
        return v;
    }
    KSA_HD int operator()(int x) const { return (int)(((uint32_t)(((uint64_t)(uint32_t)x * mul) >> 32) + (uint32_t)x) >> shift); }
};

// Whether a sequence can have the packed rows [row0, r1), the first of them its row `first` (at most 2^30 rows a sequence).
template <class A> KSA_HD bool paged_lengths_ok(const A& a, int row0, int r1, int first)
{
    return row0 >= 0 && r1 >= row0 && r1 <= a.rows && first >= 0 && r1 - row0 <= (1 << 30) && first <= (1 << 30) - (r1 - row0);
}
// A page-table entry: the page, -1 (given back) or -2 (no page of the pool).
template <class A> KSA_HD int paged_entry(const A& a, int entry) { return entry >= -1 && entry < a.num_pages ? entry : -2; }

// A row of Eq. 1: text or summary, and its number among those.
template <class A> KSA_HD int paged_place(const A& a, int row, bool& summ)
{
    const int c = a.by_chunk(row), r = row - c * (a.kk + a.m);
    summ = r >= a.kk;
    return summ ? c * a.m + (r - a.kk) : c * a.kk + r;
}
// Text tokens (summaries) among the first `row` rows of a sequence.
template <class A> KSA_HD int paged_texts(const A& a, int row)
{
    const int c = a.by_chunk(row), r = row - c * (a.kk + a.m);
    return c * a.kk + (r < a.kk ? r : a.kk);
}

// A query tile: tokens_per_tile (or fewer) consecutive text tokens, or consecutive summaries, of one sequence, or all of its rows
// of the call as they come (`mixed`).  The tile's own rows are (token, query head of the group), and what one sees is one range
// of text and one of summaries.
struct PagedTile {
    int b;                   // sequence; -1: no such tile
    bool summ, mixed;
    int x0, n;               // first text token (summary; mixed: the sequence's row `first`) and how many
    int64_t row0;            // packed row of the sequence's row `first`
    int first;
};

// Token i of a tile: its packed row, whether it is a summary, and its number among the sequence's summaries (text tokens).
template <class A> KSA_HD int paged_token(const A& a, const PagedTile& t, int i, bool& summ)
{
    if (t.mixed) return paged_place(a, t.first + i, summ);
    summ = t.summ;
    return t.x0 + i;
}
// The packed row of a tile's text token (summary) x.
template <class A> KSA_HD int64_t paged_row(const A& a, const PagedTile& t, int x)
{
    const int64_t s = a.kk + a.m;
    const int c = t.summ ? a.by_m(x) : a.by_k(x);
    const int64_t row = t.summ ? c * s + a.kk + (x - c * a.m) : c * s + (x - c * a.kk);
    return t.row0 + (row - t.first);
}

// What text token (summary) x sees: text [t_lo, t_hi), summaries [s_lo, s_hi).
struct PagedView { int t_lo, t_hi, s_lo, s_hi; };
template <class A> KSA_HD PagedView paged_view(const A& a, bool summ, int x)
{
    PagedView w;
    if (!summ) {                                       // Eq. 3
        const int c = a.by_k(x), far = c > a.C ? c - a.C : 0;
        w.t_lo = far * a.kk; w.t_hi = x + 1;
        w.s_lo = 0; w.s_hi = far * a.m;
    } else {                                           // own chunk (Sec. 2.2.1)
        const int c = a.by_m(x);
        w.t_lo = c * a.kk; w.t_hi = w.t_lo + a.kk;
        w.s_lo = c * a.m;
        w.s_hi = (a.flags & KSA_FLAG_SUMMARY_TEXT_ONLY) ? w.s_lo : x + 1;
    }
    return w;
}
// What anything in the tile sees: both ranges start with those of its first row and end with those of its last.
template <class A> KSA_HD PagedView paged_tile_view(const A& a, const PagedTile& t)
{
    const PagedView lo = paged_view(a, t.summ, t.x0), hi = paged_view(a, t.summ, t.x0 + t.n - 1);
    const bool none = t.summ && (a.flags & KSA_FLAG_SUMMARY_TEXT_ONLY);
    return PagedView{lo.t_lo, hi.t_hi, lo.s_lo, hi.s_hi > lo.s_lo && !none ? hi.s_hi : lo.s_lo};
}

// What the rows [first, first + n) of a sequence, n >= 1, see of its text (summaries): [lo, hi) but for [gap_lo, gap_hi).
struct PagedRange { int lo, hi, gap_lo, gap_hi; };
template <class A> KSA_HD PagedRange paged_range(const A& a, int first, int n, bool summ)
{
    const int t0 = paged_texts(a, first), t1 = paged_texts(a, first + n), s0 = first - t0, s1 = first + n - t1;
    const bool texts = t1 > t0, summs = s1 > s0;
    PagedRange r{0, 0, 0, 0};
    if (!summ) {
        const PagedView x = paged_view(a, !texts, texts ? t0 : s0);
        r.lo = x.t_lo;
        if (texts && summs) {                          // a first summary's chunk may start before the first text token's window
            const int lo = paged_view(a, true, s0).t_lo;
            if (lo < r.lo) r.lo = lo;
        }
        r.hi = t1;                                     // (the chunk of the last summary has ended before)
    } else {
        if (texts) r.hi = paged_view(a, false, t1 - 1).s_hi;
        if (summs && !(a.flags & KSA_FLAG_SUMMARY_TEXT_ONLY)) {
            const int lo = paged_view(a, true, s0).s_lo;
            if (!texts || r.hi == 0) r.lo = lo;
            else if (lo > r.hi) { r.gap_lo = r.hi; r.gap_hi = lo; }
            if (s1 > r.hi) r.hi = s1;
        }
    }
    return r;
}

// The key tiles (kTile rows each, from multiples of it) that hold what a query tile sees: those of the summaries, but for the
// ones inside a gap, then those of the text; part `split` of `parts` of them, [j0, j1).
template <int kTile> struct PagedWalk {
    PagedRange summ, text;
    int a0, na, b0, nb, t0, j0, j1;
    template <class A> KSA_HD void init(const A& a, const PagedTile& t, int split, int parts)
    {
        if (t.mixed) {
            text = paged_range(a, t.first, t.n, false);
            summ = paged_range(a, t.first, t.n, true);
        } else {
            const PagedView v = paged_tile_view(a, t);
            text = PagedRange{v.t_lo, v.t_hi, 0, 0};
            summ = PagedRange{v.s_lo, v.s_hi, 0, 0};
        }
        const bool gap = summ.gap_hi > summ.gap_lo;
        const int a_hi = gap ? summ.gap_lo : summ.hi;
        a0 = summ.lo / kTile;
        na = a_hi > summ.lo ? (a_hi + kTile - 1) / kTile - a0 : 0;
        b0 = gap ? summ.gap_hi / kTile : 0;
        if (gap && b0 < a0 + na) b0 = a0 + na;                     // (a tile that holds rows from both sides comes once)
        nb = gap && (summ.hi + kTile - 1) / kTile > b0 ? (summ.hi + kTile - 1) / kTile - b0 : 0;
        t0 = text.lo / kTile;
        const int tiles = na + nb + (text.hi + kTile - 1) / kTile - t0, per = (tiles + parts - 1) / parts;
        j0 = split * per < tiles ? split * per : tiles;
        j1 = j0 + per < tiles ? j0 + per : tiles;
    }
    // Tile j: its stream, its first row, and what of the stream is seen
    struct Tile {
        bool summ;
        int x0;
        PagedRange see;
        KSA_HD bool sees(int x) const { return x >= see.lo && x < see.hi && !(x >= see.gap_lo && x < see.gap_hi); }
        // any of the rows [x, x + n); all of the tile's
        KSA_HD bool sees_any(int x, int n) const { return x < see.hi && x + n > see.lo && !(x >= see.gap_lo && x + n <= see.gap_hi); }
        KSA_HD bool sees_all() const { return x0 >= see.lo && x0 + kTile <= see.hi && !(x0 < see.gap_hi && x0 + kTile > see.gap_lo); }
    };
    KSA_HD Tile at(int j) const
    {
        if (j < na + nb) return Tile{true, (j < na ? a0 + j : b0 + j - na) * kTile, summ};
        return Tile{false, (t0 + j - na - nb) * kTile, text};
    }
};

}  // namespace ksa
