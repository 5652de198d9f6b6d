// The paged KV cache: rows written into their pages (quantised on the way) and read back, and the C ABI of the paged calls.
//
// Both passes are bound by HBM: an element is read and written once.  D / 8 lanes take one row of one head, 16 bytes of
// bf16 each, K and V of it at once; the row's sequence, page and place in the page are worked out by every lane for itself.
// Measured: 32,176 bf16 rows of 16 heads of 128 written in 84.6 us = 6,230 GB/s, 147,456 e4m3 rows of 4 heads read back in 75.6 - 79 us =
// 6,010 - 5,750 GB/s (a copy: 6,465); 9,216 e4m3 rows of 8 heads written in 13.6 us, where launch and dependent loads count.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "ksa_host.h"
#include "ksa_launch.h"
#include "ksa_paged.h"
#include "ksa_ptx.cuh"

namespace ksa {

// (9,216 rows of 8 heads appended in 8 bits by blocks of 128, 256, 512 threads: 15.5, 16.9, 17.9 us; reading back moves less)
constexpr int kRowThreads = 128;
constexpr int kUnpackThreads = 256;

// A lane's sequence among up to 32: where its rows start, how many are cached; where the last one's end
struct PagedSeqs { int mine, rows, end; };
__device__ __forceinline__ PagedSeqs paged_seqs(const PagedArgs& a)
{
    PagedSeqs s{};
    if (a.B <= 32) {
        const int lane = threadIdx.x & 31;
        s.mine = __ldcg(a.cu + min(lane, a.B)); s.rows = __ldcg(a.cached + min(lane, a.B - 1)); s.end = __ldcg(a.cu + a.B);
    }
    return s;
}
// Where packed row i of the call lies: its page (or -1, -2) and the place in it; false if it is no row of a sequence.
// Executed by whole warps.  Up to 32 sequences are searched in registers (one load instead of one after another), as many steps as
// their number needs.
__device__ __forceinline__ bool paged_find(const PagedArgs& a, const PagedSeqs& seqs, int i, int& page, int& slot)
{
    int lo = 0, hi = a.B - 1, row0, r1, first;                 // the last sequence that starts at or before row i
    if (a.B <= 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (a.B <= o) continue;
            const int at = __shfl_sync(0xffffffffu, seqs.mine, (lo + o) & 31);
            if (lo + o <= hi && at <= i) lo += o;
        }
        row0 = __shfl_sync(0xffffffffu, seqs.mine, lo);
        r1 = __shfl_sync(0xffffffffu, seqs.mine, (lo + 1) & 31);
        if (lo == 31) r1 = seqs.end;
        first = __shfl_sync(0xffffffffu, seqs.rows, lo);
    } else {
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldcg(a.cu + mid) <= i) lo = mid; else hi = mid - 1;
        }
        row0 = __ldcg(a.cu + lo);
        r1 = __ldcg(a.cu + lo + 1);
        first = __ldcg(a.cached + lo);
    }
    int n;
    if (i >= a.rows || !paged_seq(a, lo, row0, r1, first, n) || i < row0 || i >= r1) return false;
    bool summ;
    const int x = paged_place(a, first + (i - row0), summ);
    page = paged_page(a, lo, summ, x);
    slot = x & ((1 << a.page_shift) - 1);
    return true;
}

// Whether a place is one of the pool (KSA_DEBUG builds: recorded, and the access skipped)
__device__ __forceinline__ bool paged_place_ok(const PagedArgs& a, int page, int h, int slot)
{
    return ksa_in_bounds(page >= 0 && page < a.num_pages && h < a.Hkv && slot >= 0 && slot < (1 << a.page_shift), a.status);
}

// Every sequence's lengths, looked at by the first block: a row's search meets only those of the sequences that it lands in.
__device__ __forceinline__ void paged_check_all(const PagedArgs& a)
{
    if (blockIdx.x + blockIdx.y != 0) return;
    for (int b = threadIdx.x; b < a.B; b += kRowThreads) {
        int n;
        paged_seq(a, b, __ldcg(a.cu + b), __ldcg(a.cu + b + 1), __ldcg(a.cached + b), n);
    }
}

// 8 bf16 values times a power of two -> 8 e4m3
__device__ __forceinline__ uint32_t e4m3x2_from_f32(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint2 quantise8(const uint4& x, float f)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = e4m3x2_from_f32(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
    return make_uint2(y[0] | (y[1] << 16), y[2] | (y[3] << 16));
}
// The largest scale, 2^120: 256 times it is more than bf16 holds, the value below it is 240 (0x77)
__device__ __forceinline__ uint2 keep_finite(const uint2& y)
{
    auto cut = [](uint32_t w) { return __vminu4(w & 0x7f7f7f7fu, 0x77777777u) | (w & 0x80808080u); };
    return make_uint2(cut(y.x), cut(y.y));
}
// largest magnitude of 8 bf16 values, as bits (in both halves' order: an infinity or a NaN comes out at 0x7f80 or above)
__device__ __forceinline__ uint32_t top8(const uint4& x)
{
    const uint32_t m = 0x7fff7fffu;
    const uint32_t t = __vmaxu2(__vmaxu2(x.x & m, x.y & m), __vmaxu2(x.z & m, x.w & m));
    return max(t >> 16, t & 0xffffu);
}

// A thread's unit is a row and kHeads of its heads: one search for the row's place, then 2 kHeads loads in flight (1, 2, 4, 8
// heads: 147,456 e4m3 rows of 4 heads read back in 158, 98, 76, 85 us; 32 rows appended by 1, 2, 8 in 2.0, 2.5, 3.5 us).
template <int D, bool E4M3, int kHeads>
__global__ void __launch_bounds__(kRowThreads) ksa_paged_append_kernel(PagedArgs a)
{
    constexpr int kLanes = D / 8, kUnits = kRowThreads / kLanes;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int lane = threadIdx.x % kLanes, i = blockIdx.x * kUnits + threadIdx.x / kLanes, h0 = blockIdx.y * kHeads;
    // The rows' values need no place to be loaded, and the search's loads come back sooner without them in front.  9,216 e4m3 rows of 8
    // heads, the values asked for first, between the lengths and the search, after it: 15.5, 14.5, 13.7 us; 32 rows: 2.15, 2.00,
    // 2.4; 33,000 bf16 rows of 16 heads: 86.5, 84.6, 85.4.
    constexpr bool kSearchFirst = E4M3 && kHeads > 1;
    const PagedSeqs seqs = paged_seqs(a);
    int page = -1, slot = 0;
    bool put = false;
    if constexpr (kSearchFirst) put = paged_find(a, seqs, i, page, slot);
    uint4 xk[kHeads], xv[kHeads];
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
        xk[c] = xv[c] = uint4{};
        if (i < a.rows && h0 + c < a.Hkv) {
            xk[c] = __ldcg(reinterpret_cast<const uint4*>(a.k + i * a.k_st + (h0 + c) * a.k_sh + lane * 8));
            xv[c] = __ldcg(reinterpret_cast<const uint4*>(a.v + i * a.v_st + (h0 + c) * a.v_sh + lane * 8));
        }
    }
    if constexpr (!kSearchFirst) put = paged_find(a, seqs, i, page, slot);
    if (put && page < 0) {
        atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_PAGE);
        put = false;
    }
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
        const int h = h0 + c;
        const int64_t at = page * a.page_st + h * a.head_st + slot * a.row_st;
        if constexpr (!E4M3) {
            if (!put || h >= a.Hkv || !paged_place_ok(a, page, h, slot)) continue;
            *reinterpret_cast<uint4*>(a.kp + at + lane * 16) = xk[c];
            *reinterpret_cast<uint4*>(a.vp + at + lane * 16) = xv[c];
        } else {
            uint32_t top = top8(xk[c]) | (top8(xv[c]) << 16);  // K's in the low half, V's in the high half
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (!put || h >= a.Hkv || !paged_place_ok(a, page, h, slot)) continue;
            // the row's largest magnitude is (1 + mant / 128) 2^(e - 127): within 448 = 1.75 * 2^8 at 2^(e - 135), or at twice that
            auto scale_of = [](uint32_t t) { return t >= 0x7f80u ? 255 : max(17, (int)(t >> 7) - 8 + ((t & 0x7fu) > 0x60u)); };
            const int ek = scale_of(top & 0xffffu), ev = scale_of(top >> 16);
            // (two to the minus that is a normal number for every byte from 17 to 247)
            uint2 yk = quantise8(xk[c], __uint_as_float((uint32_t)(254 - ek) << 23)), yv = quantise8(xv[c], __uint_as_float((uint32_t)(254 - ev) << 23));
            if (ek == 247) yk = keep_finite(yk);
            if (ev == 247) yv = keep_finite(yv);
            *reinterpret_cast<uint2*>(a.kp + at + lane * 8) = ek == 255 ? make_uint2(0, 0) : yk;
            *reinterpret_cast<uint2*>(a.vp + at + lane * 8) = ev == 255 ? make_uint2(0, 0) : yv;
            if (lane == 0) {
                const int64_t se = (((int64_t)page * a.Hkv + h) << a.page_shift) + slot;
                a.ke[se] = (uint8_t)ek;
                a.ve[se] = (uint8_t)ev;
            }
        }
    }
    paged_check_all(a);
}

template <int D, bool E4M3, int kHeads>
__global__ void __launch_bounds__(kRowThreads) ksa_paged_gather_kernel(PagedArgs a)
{
    constexpr int kLanes = D / 8, kUnits = kRowThreads / kLanes;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int lane = threadIdx.x % kLanes, i = blockIdx.x * kUnits + threadIdx.x / kLanes, h0 = blockIdx.y * kHeads;
    int page = -1, slot = 0;
    const PagedSeqs seqs = paged_seqs(a);
    const bool row = paged_find(a, seqs, i, page, slot);
    paged_check_all(a);
    if (!row) return;
    if (page == -2) atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_PAGE);
    using Raw = typename std::conditional<E4M3, uint2, uint4>::type;
    Raw yk[kHeads], yv[kHeads];
    uint32_t ek[kHeads], ev[kHeads];
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
        yk[c] = yv[c] = Raw{};
        ek[c] = ev[c] = 0;
        const int h = h0 + c;
        if (page >= 0 && h < a.Hkv && paged_place_ok(a, page, h, slot)) {
            const int64_t at = page * a.page_st + h * a.head_st + slot * a.row_st + lane * (int)sizeof(Raw);
            yk[c] = __ldcg(reinterpret_cast<const Raw*>(a.kp + at));
            yv[c] = __ldcg(reinterpret_cast<const Raw*>(a.vp + at));
            if constexpr (E4M3) {
                const int64_t se = (((int64_t)page * a.Hkv + h) << a.page_shift) + slot;
                ek[c] = __ldcg(a.ke + se); ev[c] = __ldcg(a.ve + se);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
        const int h = h0 + c;
        if (h >= a.Hkv || !ksa_in_bounds(i >= 0 && i < a.rows, a.status)) continue;
        uint4 xk, xv;
        if constexpr (E4M3) {
            const float fk = e8m0_scale(ek[c]), fv = e8m0_scale(ev[c]);
            auto two = [](uint32_t y, float f) { const float2 v = e4m3x2_to_f32(y & 0xffffu); return ptx::pack_bf16x2(v.x * f, v.y * f); };
            xk = make_uint4(two(yk[c].x, fk), two(yk[c].x >> 16, fk), two(yk[c].y, fk), two(yk[c].y >> 16, fk));
            xv = make_uint4(two(yv[c].x, fv), two(yv[c].x >> 16, fv), two(yv[c].y, fv), two(yv[c].y >> 16, fv));
        } else { xk = yk[c]; xv = yv[c]; }
        *reinterpret_cast<uint4*>(a.k + i * a.k_st + h * a.k_sh + lane * 8) = xk;
        *reinterpret_cast<uint4*>(a.v + i * a.v_st + h * a.v_sh + lane * 8) = xv;
    }
}

// ---- e4m3 rows in view as bf16 pages of 128 rows ----------------------------------------------------------------------------
// For calls with many query rows a sequence: the attention kernel on bf16 pages converts nothing, while the one on e4m3
// pages converts a key tile again for every 256 query rows.  One block per page of the copy (128 text tokens or summaries from a
// multiple of 128) and KV head; the copy's page tables are written on the way.  Only rows that some row of the call sees are
// read (and their pages looked up); the others' places stay as they are, as in any page.
struct UnpackArgs {
    uint16_t* k; uint16_t* v;                        // [batch * seq_pages][Hkv][128][D]
    int32_t* text_table; int32_t* summ_table;        // [batch][text_cols], [batch][summ_cols]
    int32_t text_cols, summ_cols, text_pages, seq_pages;     // text_pages: of a sequence, before its pages of summaries
};

template <int D>
__global__ void __launch_bounds__(kUnpackThreads) ksa_paged_unpack_kernel(PagedArgs a, UnpackArgs u)
{
    constexpr int kLanes = D / 16, kRowsPass = kUnpackThreads / kLanes;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int b = blockIdx.z, h = blockIdx.y, slot = blockIdx.x;
    int n;
    const int first = __ldcg(a.cached + b);
    if (!paged_seq(a, b, __ldcg(a.cu + b), __ldcg(a.cu + b + 1), first, n) || n < a.rows_min || n > a.rows_max) return;
    const bool summ = slot >= u.text_pages;
    const PagedRange see = paged_range(a, first, n, summ);
    const int tile = summ ? slot - u.text_pages : see.lo / 128 + slot, x0 = tile * 128;
    if (x0 >= see.hi || x0 + 128 <= see.lo || tile >= (summ ? u.summ_cols : u.text_cols)) return;
    const int page = b * u.seq_pages + slot;
    if (!ksa_in_bounds(tile >= 0 && slot < u.seq_pages && h < a.Hkv && b < a.B, a.status)) return;
    if (h == 0 && threadIdx.x == 0) (summ ? u.summ_table : u.text_table)[(int64_t)b * (summ ? u.summ_cols : u.text_cols) + tile] = page;
    // all of a thread's page lookups, then all of its loads, then its stores
    constexpr int kPasses = 128 / kRowsPass;
    const int lane = threadIdx.x % kLanes, in_page = (1 << a.page_shift) - 1;
    int from[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int x = x0 + threadIdx.x / kLanes + i * kRowsPass;
        from[i] = x < see.lo || x >= see.hi || (x >= see.gap_lo && x < see.gap_hi) ? -3 : paged_page(a, b, summ, x);
    }
    uint4 yk[kPasses], yv[kPasses];
    uint32_t ek[kPasses], ev[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (from[i] < 0) {
            if (from[i] != -3) atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_PAGE);
            continue;
        }
        const int in = x0 + threadIdx.x / kLanes + i * kRowsPass & in_page;
        if (!paged_place_ok(a, from[i], h, in)) { from[i] = -3; continue; }
        const int64_t at = from[i] * a.page_st + h * a.head_st + in * a.row_st + lane * 16, se = (((int64_t)from[i] * a.Hkv + h) << a.page_shift) + in;
        yk[i] = __ldcg(reinterpret_cast<const uint4*>(a.kp + at)); yv[i] = __ldcg(reinterpret_cast<const uint4*>(a.vp + at));
        ek[i] = __ldcg(a.ke + se); ev[i] = __ldcg(a.ve + se);
    }
    auto put = [](uint16_t* dst, const uint4& y, float f) {
        uint4 z[2];
        uint32_t* w = reinterpret_cast<uint32_t*>(z);
        const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = e4m3x2_to_f32(yw[i] & 0xffffu), q = e4m3x2_to_f32(yw[i] >> 16);
            w[2 * i] = ptx::pack_bf16x2(p.x * f, p.y * f); w[2 * i + 1] = ptx::pack_bf16x2(q.x * f, q.y * f);
        }
        reinterpret_cast<uint4*>(dst)[0] = z[0]; reinterpret_cast<uint4*>(dst)[1] = z[1];
    };
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (from[i] < 0) continue;
        const int64_t to = (((int64_t)page * a.Hkv + h) * 128 + threadIdx.x / kLanes + i * kRowsPass) * D + lane * 16;
        put(u.k + to, yk[i], e8m0_scale(ek[i]));
        put(u.v + to, yv[i], e8m0_scale(ev[i]));
    }
}

// Where things stand in the workspace of a call, and its size; 0 bytes where the call makes no copy.
struct UnpackLayout { int64_t text_cols, summ_cols, text_pages, seq_pages, kv_bytes, tables, bytes; };
static UnpackLayout unpack_layout(const ksa_paged_params* p)
{
    UnpackLayout l{};
    const int64_t G = p->num_q_heads / p->num_kv_heads;
    // From 1,024 query rows (four tiles of 256) a sequence on: the tcgen05 kernel converts a key tile once for each of them.  256 rows over
    // 36,864, 32/8 heads: 65 us without the copy, 59 with it; 128 rows: 43 and 46; 1,152: 122 and 89.
    if (p->kv_format != KSA_KV_E4M3 || p->num_rows * G < 1024 * (int64_t)p->batch || (p->flags & KSA_FLAG_PAGED_MMA_SYNC)) return l;
    const int64_t text = (int64_t)p->text_cols * p->page_rows, summ = p->summaries_per_chunk > 0 ? (int64_t)p->summ_cols * p->page_rows : 0;
    l.text_cols = (text + 127) / 128; l.summ_cols = (summ + 127) / 128;
    const int64_t seen = ((int64_t)p->window_chunks + 2) * p->chunk_len + p->num_rows;        // text tokens in view, at most
    l.text_pages = std::min(l.text_cols, seen / 128 + 2);
    l.seq_pages = l.text_pages + l.summ_cols;
    l.kv_bytes = p->batch * l.seq_pages * p->num_kv_heads * 128 * p->head_dim * 2;
    l.tables = 2 * l.kv_bytes;
    l.bytes = l.tables + (l.text_cols + l.summ_cols) * p->batch * 4;
    if (l.bytes > (2ll << 30) || p->batch * l.seq_pages > (1 << 30)) return UnpackLayout{};
    return l;
}

// Four heads a thread, or one where that leaves SMs without a block
template <class F>
static cudaError_t launch_rows(const PagedArgs& a, F kernel_for, int num_sms, cudaStream_t stream)
{
    const int per = kRowThreads / (a.D / 8), blocks = (a.rows + per - 1) / per;
    const int heads = (int64_t)blocks * a.Hkv <= 2 * num_sms ? 1 : 4;
    return launch_dependent(kernel_for(heads == 1), dim3((unsigned)blocks, (unsigned)((a.Hkv + heads - 1) / heads)), kRowThreads, 0, stream, a);
}
cudaError_t launch_paged_append(const PagedArgs& a, bool e4m3, int num_sms, cudaStream_t stream)
{
    return launch_rows(a, [&](bool one) {
        if (a.D == 128) return e4m3 ? one ? ksa_paged_append_kernel<128, true, 1> : ksa_paged_append_kernel<128, true, 4> : one ? ksa_paged_append_kernel<128, false, 1> : ksa_paged_append_kernel<128, false, 4>;
        return e4m3 ? one ? ksa_paged_append_kernel<64, true, 1> : ksa_paged_append_kernel<64, true, 4> : one ? ksa_paged_append_kernel<64, false, 1> : ksa_paged_append_kernel<64, false, 4>;
    }, num_sms, stream);
}
cudaError_t launch_paged_gather(const PagedArgs& a, bool e4m3, int num_sms, cudaStream_t stream)
{
    return launch_rows(a, [&](bool one) {
        if (a.D == 128) return e4m3 ? one ? ksa_paged_gather_kernel<128, true, 1> : ksa_paged_gather_kernel<128, true, 4> : one ? ksa_paged_gather_kernel<128, false, 1> : ksa_paged_gather_kernel<128, false, 4>;
        return e4m3 ? one ? ksa_paged_gather_kernel<64, true, 1> : ksa_paged_gather_kernel<64, true, 4> : one ? ksa_paged_gather_kernel<64, false, 1> : ksa_paged_gather_kernel<64, false, 4>;
    }, num_sms, stream);
}

}  // namespace ksa

// =================================================================================================
// C ABI
// =================================================================================================
using namespace ksa;

#define KSA_API extern "C" __attribute__((visibility("default")))

static int validate_shape(const ksa_paged_params* p)
{
    if (!p || p->struct_size != (int32_t)sizeof(ksa_paged_params)) return KSA_ERR_INVALID_ARG;
    if (p->batch < 1 || p->num_rows < 0 || p->chunk_len < 1 || p->summaries_per_chunk < 0 || p->window_chunks < 0) return KSA_ERR_INVALID_ARG;
    if (p->num_q_heads < 1 || p->num_kv_heads < 1 || p->num_q_heads % p->num_kv_heads != 0) return KSA_ERR_INVALID_ARG;
    if (!(p->softmax_scale > 0.f) || p->softmax_scale > 1e30f) return KSA_ERR_INVALID_ARG;
    constexpr uint32_t kOne = KSA_FLAG_PAGED_MMA_SYNC | KSA_FLAG_PAGED_TCGEN05;
    if (p->flags & ~(KSA_FLAG_SUMMARY_TEXT_ONLY | kOne) || (p->flags & kOne) == kOne) return KSA_ERR_INVALID_ARG;
    if (p->kv_format != KSA_KV_BF16 && p->kv_format != KSA_KV_E4M3) return KSA_ERR_INVALID_ARG;
    if (p->num_pages < 1 || p->text_cols < 1 || p->summ_cols < (p->summaries_per_chunk > 0 ? 1 : 0)) return KSA_ERR_INVALID_ARG;
    if (p->head_dim != 64 && p->head_dim != 128) return KSA_ERR_UNSUPPORTED;
    if (p->page_rows != 16 && p->page_rows != 32 && p->page_rows != 64 && p->page_rows != 128) return KSA_ERR_UNSUPPORTED;
    if (p->num_q_heads / p->num_kv_heads > 64 || p->num_q_heads > 1024 || p->batch > 65535 || p->num_rows > (1 << 24)) return KSA_ERR_UNSUPPORTED;
    if ((int64_t)p->chunk_len + p->summaries_per_chunk > (1 << 30)) return KSA_ERR_UNSUPPORTED;
    return KSA_OK;
}

static int validate_pool_strides(const ksa_paged_params* p)
{
    const int64_t unit = p->kv_format == KSA_KV_BF16 ? 8 : 16;              // 16 bytes
    auto stride_of = [&](int64_t st) { return st <= 0 || st % unit != 0 ? KSA_ERR_INVALID_ARG : st >= (1ll << 38) ? KSA_ERR_UNSUPPORTED : KSA_OK; };
    int rc = p->row_stride < p->head_dim ? KSA_ERR_INVALID_ARG : stride_of(p->row_stride);
    if (rc == KSA_OK && p->num_kv_heads > 1) rc = stride_of(p->head_stride);             // (of one head, of one page: any)
    if (rc == KSA_OK && p->num_pages > 1) rc = stride_of(p->page_stride);
    return rc;
}

static int validate_paged(const ksa_paged_params* p, const ksa_paged_kv* kv)
{
    int rc = validate_shape(p);
    if (rc == KSA_OK) rc = validate_pool_strides(p);
    if (rc != KSA_OK) return rc;
    if (!kv) return KSA_ERR_INVALID_ARG;
    auto misaligned = [](const void* q) { return ((uintptr_t)q & 15) != 0; };
    if (!kv->kpages || !kv->vpages || misaligned(kv->kpages) || misaligned(kv->vpages)) return KSA_ERR_INVALID_ARG;
    if (p->kv_format == KSA_KV_E4M3 && (!kv->kscale || !kv->vscale || misaligned(kv->kscale) || misaligned(kv->vscale))) return KSA_ERR_INVALID_ARG;
    if (!kv->text_table || (!kv->summ_table && p->summaries_per_chunk > 0) || !kv->cached || !kv->cu_rows) return KSA_ERR_INVALID_ARG;
    for (const int32_t* t : {kv->text_table, kv->summ_table, kv->cached, kv->cu_rows})
        if ((uintptr_t)t & 3) return KSA_ERR_INVALID_ARG;
    return KSA_OK;
}

// A packed tensor of the call; one that is written has a place for every row and head
static bool tensor_ok(const void* t, int64_t st, int64_t sh)
{
    return t && ((uintptr_t)t & 15) == 0 && st >= 0 && sh >= 0 && st % 8 == 0 && sh % 8 == 0 && st < (1ll << 38) && sh < (1ll << 38);
}
static bool written_ok(const void* t, int64_t st, int64_t sh, int rows, int heads)
{
    return tensor_ok(t, st, sh) && (rows == 1 || st > 0) && (heads == 1 || sh > 0);
}

static PagedArgs paged_args(ksa_ctx* ctx, const ksa_paged_kv* kv, const ksa_paged_params* p)
{
    PagedArgs a{};
    a.kp = (uint8_t*)kv->kpages; a.vp = (uint8_t*)kv->vpages; a.ke = kv->kscale; a.ve = kv->vscale;
    a.text_table = kv->text_table; a.summ_table = kv->summ_table; a.cached = kv->cached; a.cu = kv->cu_rows;
    const int64_t width = p->kv_format == KSA_KV_BF16 ? 2 : 1;
    a.page_st = p->num_pages > 1 ? p->page_stride * width : 0; a.head_st = p->num_kv_heads > 1 ? p->head_stride * width : 0;
    a.row_st = p->row_stride * width;
    a.q_st = p->q_stride_tok; a.q_sh = p->q_stride_head; a.k_st = p->k_stride_tok; a.k_sh = p->k_stride_head;
    a.v_st = p->v_stride_tok; a.v_sh = p->v_stride_head; a.o_st = p->o_stride_tok; a.o_sh = p->o_stride_head;
    a.B = p->batch; a.rows = p->num_rows; a.kk = p->chunk_len; a.m = p->summaries_per_chunk; a.C = p->window_chunks;
    a.Hq = p->num_q_heads; a.Hkv = p->num_kv_heads; a.G = a.Hq / a.Hkv; a.D = p->head_dim;
    a.by_chunk = PagedDiv::by(a.kk + a.m); a.by_k = PagedDiv::by(a.kk); a.by_m = PagedDiv::by(a.m);
    a.page_shift = p->page_rows == 16 ? 4 : p->page_rows == 32 ? 5 : p->page_rows == 64 ? 6 : 7;
    a.num_pages = p->num_pages; a.text_cols = p->text_cols; a.summ_cols = p->summ_cols;
    a.flags = p->flags;
    a.scale_log2 = p->softmax_scale * 1.4426950408889634f;
    a.status = ksa_ctx_status_word(ctx);
    return a;
}

namespace {
// The context's device for the length of a call
struct OnDevice {
    int before = -1;
    cudaError_t err;
    explicit OnDevice(int device)
    {
        err = cudaGetDevice(&before);
        if (err == cudaSuccess && before != device) err = cudaSetDevice(device); else before = -1;
    }
    ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
};
}  // namespace

template <class F>
static int paged_call(ksa_ctx* ctx, F launch)
{
    OnDevice on(ksa_ctx_device(ctx));
    cudaError_t e = on.err;
    if (e == cudaSuccess) e = launch();
    if (e != cudaSuccess) return ksa_ctx_cuda_fail(ctx, (int)e);
    ksa_ctx_add_launches(ctx, 1);
    return KSA_OK;
}

KSA_API int ksa_paged_append(ksa_ctx* ctx, const ksa_paged_kv* kv, const void* k, const void* v, const ksa_paged_params* p, void* cuda_stream)
{
    const int rc = validate_paged(p, kv);
    if (rc != KSA_OK) return rc;
    if (!ctx) return KSA_ERR_INVALID_ARG;
    if (p->num_rows == 0) return KSA_OK;
    if (!tensor_ok(k, p->k_stride_tok, p->k_stride_head) || !tensor_ok(v, p->v_stride_tok, p->v_stride_head)) return KSA_ERR_INVALID_ARG;
    PagedArgs a = paged_args(ctx, kv, p);
    a.k = (uint16_t*)k; a.v = (uint16_t*)v;
    return paged_call(ctx, [&] { return launch_paged_append(a, p->kv_format == KSA_KV_E4M3, ksa_ctx_num_sms(ctx), (cudaStream_t)cuda_stream); });
}

KSA_API int ksa_paged_gather(ksa_ctx* ctx, const ksa_paged_kv* kv, void* k, void* v, const ksa_paged_params* p, void* cuda_stream)
{
    const int rc = validate_paged(p, kv);
    if (rc != KSA_OK) return rc;
    if (!ctx) return KSA_ERR_INVALID_ARG;
    if (p->num_rows == 0) return KSA_OK;
    if (!written_ok(k, p->k_stride_tok, p->k_stride_head, p->num_rows, p->num_kv_heads) || !written_ok(v, p->v_stride_tok, p->v_stride_head, p->num_rows, p->num_kv_heads))
        return KSA_ERR_INVALID_ARG;
    PagedArgs a = paged_args(ctx, kv, p);
    a.k = (uint16_t*)k; a.v = (uint16_t*)v;
    return paged_call(ctx, [&] { return launch_paged_gather(a, p->kv_format == KSA_KV_E4M3, ksa_ctx_num_sms(ctx), (cudaStream_t)cuda_stream); });
}

KSA_API int ksa_paged_workspace_bytes(const ksa_paged_params* p, size_t* bytes)
{
    if (!bytes) return KSA_ERR_INVALID_ARG;
    const int rc = validate_shape(p);
    if (rc != KSA_OK) return rc;
    *bytes = (size_t)unpack_layout(p).bytes;
    return KSA_OK;
}

KSA_API int ksa_paged_attn(ksa_ctx* ctx, const ksa_paged_kv* kv, const void* q, void* out, float* lse, void* workspace, size_t workspace_bytes,
                           const ksa_paged_params* p, void* cuda_stream)
{
    const int rc = validate_paged(p, kv);
    if (rc != KSA_OK) return rc;
    if (!ctx) return KSA_ERR_INVALID_ARG;
    if (p->num_rows == 0) return KSA_OK;
    if (!tensor_ok(q, p->q_stride_tok, p->q_stride_head) || !written_ok(out, p->o_stride_tok, p->o_stride_head, p->num_rows, p->num_q_heads) || !lse || ((uintptr_t)lse & 3)) return KSA_ERR_INVALID_ARG;
    if (workspace && ((uintptr_t)workspace & 255)) return KSA_ERR_INVALID_ARG;
    PagedArgs a = paged_args(ctx, kv, p);
    a.q = (const uint16_t*)q; a.out = (uint16_t*)out; a.lse = lse;
    bool e4m3 = p->kv_format == KSA_KV_E4M3;
    return paged_call(ctx, [&]() -> cudaError_t {
        const PagedEncode encode = (PagedEncode)ksa_ctx_encode_tiled(ctx);
        const cudaStream_t stream = (cudaStream_t)cuda_stream;
        cudaError_t e = (cudaError_t)ksa_ctx_paged_setup(ctx, [] {
            const cudaError_t e = setup_paged_attn();
            return (int)(e == cudaSuccess ? setup_paged_tc() : e);
        });
        if (e != cudaSuccess) return e;
        // Up to 16 query rows a sequence, on average (64 over e4m3 pages): the mma.sync kernel for all.  16 sequences of 3, 4, 5, 6, 8 rows
        // over 800 to 37,000, 32/8 heads (12 to 32 query rows), that one and the tcgen05 kernel: bf16 50, 50, 55, 86, 86 and 48, 51, 51,
        // 52, 55 us, e4m3 40, 41, 48, 57, 60 and 78, 81, 82, 84, 90 us.  More: the same where it is expected to be faster, since
        // it finds work for more SMs in small calls (115 rows over 720, 4/4 heads: 8.3 and 17 us; 191 e4m3 rows over 7,000,
        // 10/2 heads: 15 and 26).  Else, with several sequences, that one for those that fit into
        // its tiles (single tokens beside prompts), and the tcgen05 kernel, which takes as long over one query row as over 256,
        // beside it for the others: 24 tokens over 90,000 to 113,000 rows and 1,152 rows over 36,864, 32/8 heads:
        // e4m3 484 -> 261 us, bf16 251 -> 259; the 24 over 1,000 to 3,500 rows: 152 -> 156, 126 -> 100.  A launch that finds no
        // such sequence costs 4 us.
        const int sms = ksa_ctx_num_sms(ctx), query_rows = (int64_t)a.rows * a.G <= 8 * (int64_t)a.B ? 8 : 16;
        const int64_t rows = (int64_t)a.rows * a.G;
        a.rows_min = 1; a.rows_max = a.rows;
        const UnpackLayout l = unpack_layout(p);
        const bool copy = l.bytes > 0 && workspace && workspace_bytes >= (size_t)l.bytes;
        bool few = rows <= (e4m3 ? 64 : 16) * (int64_t)a.B || paged_attn_us(a, e4m3, query_rows, sms) < paged_tc_us(a, e4m3 && !copy, sms) + (copy ? 6.0f : 0.0f);
        if (p->flags & (KSA_FLAG_PAGED_MMA_SYNC | KSA_FLAG_PAGED_TCGEN05)) few = p->flags & KSA_FLAG_PAGED_MMA_SYNC;
        if (few) return launch_paged_attn(a, e4m3, query_rows, sms, encode, stream);
        const int small = a.B < 4 || rows <= 64 * (int64_t)a.B || a.G > 16 ? 0 : (a.G > 8 ? 16 : 8) / a.G;      // rows of a sequence for the former
        UnpackArgs u{};
        if (copy) {
            u.k = (uint16_t*)workspace; u.v = u.k + l.kv_bytes / 2;
            u.text_table = (int32_t*)((char*)workspace + l.tables); u.summ_table = u.text_table + l.text_cols * a.B;
            u.text_cols = (int32_t)l.text_cols; u.summ_cols = (int32_t)l.summ_cols; u.text_pages = (int32_t)l.text_pages; u.seq_pages = (int32_t)l.seq_pages;
            a.rows_min = small + 1;
            e = launch_dependent(a.D == 128 ? ksa_paged_unpack_kernel<128> : ksa_paged_unpack_kernel<64>,
                                 dim3((unsigned)l.seq_pages, (unsigned)a.Hkv, (unsigned)a.B), kUnpackThreads, 0, stream, a, u);
            if (e != cudaSuccess) return e;
            ksa_ctx_add_launches(ctx, 1);
        }
        if (small > 0) {
            a.rows_min = 1; a.rows_max = small; a.beside = 1;
            if ((e = launch_paged_attn(a, e4m3, small * a.G, sms, encode, stream)) != cudaSuccess) return e;
            ksa_ctx_add_launches(ctx, 1);
            a.beside = 2;
        }
        a.rows_min = small + 1; a.rows_max = a.rows;
        if (copy) {                                            // from here on the cache is the copy
            a.kp = (uint8_t*)u.k; a.vp = (uint8_t*)u.v; a.ke = a.ve = nullptr;
            a.text_table = u.text_table; a.summ_table = u.summ_table; a.text_cols = u.text_cols; a.summ_cols = u.summ_cols;
            a.page_shift = 7; a.num_pages = (int32_t)(a.B * l.seq_pages);
            a.row_st = a.D * 2; a.head_st = 128 * a.row_st; a.page_st = a.Hkv * a.head_st;
            e4m3 = false;
        }
        return launch_paged_tc(a, e4m3, sms, encode, stream);
    });
}
