// Internal declarations of the paged KV cache: arguments of its kernels, where a row lies, which rows a query tile sees.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/ksa_paged.h"
#include "ksa_common.h"
#include "ksa_paged_index.h"

namespace ksa {

struct PagedArgs {
    uint8_t* kp; uint8_t* vp; uint8_t* ke; uint8_t* ve;              // pages (bytes), scale bytes
    const int32_t* text_table; const int32_t* summ_table; const int32_t* cached; const int32_t* cu;
    uint16_t* k; uint16_t* v;                                        // rows written or read back
    const uint16_t* q; uint16_t* out; float* lse;
    int64_t page_st, head_st, row_st;                                // of the pages, in bytes
    int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh, o_st, o_sh;          // in elements
    int32_t B, rows, kk, m, C, Hq, Hkv, G, D;
    PagedDiv by_chunk, by_k, by_m, by_tile;                          // divisors k + m, k, m, tokens_per_tile
    PagedDiv by_heads, by_group, by_split;                           // ... of a CTA's number and of a tile's row, see the kernels
    int32_t page_shift, num_pages, text_cols, summ_cols;             // page_rows = 1 << page_shift
    int32_t tokens_per_tile, head_blocks, nsplit, box_rows;        // attention: see the kernels
    int32_t rows_min, rows_max;                                      // ... of sequences with as many rows in the call
    int32_t beside;                                                  // 1: the kernel behind runs beside this one; 2: this one is it
    uint32_t flags;
    float scale_log2;
    int32_t* status;
};

cudaError_t launch_paged_append(const PagedArgs& a, bool e4m3, int num_sms, cudaStream_t stream);
cudaError_t launch_paged_gather(const PagedArgs& a, bool e4m3, int num_sms, cudaStream_t stream);
typedef CUresult (*PagedEncode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// Map of a page pool, [D, page rows, KV heads, pages] with a box of box_rows rows of box_bytes bytes of one page and head.
bool encode_pages(PagedEncode encode, CUtensorMap* map, void* base, const PagedArgs& a, bool e4m3, int box_bytes, int box_rows, CUtensorMapSwizzle swizzle);
// Tiles of up to 8 or 16 query rows (mma.sync), and of up to 256 (tcgen05).
cudaError_t launch_paged_attn(const PagedArgs& a, bool e4m3, int query_rows, int num_sms, PagedEncode encode, cudaStream_t stream);
cudaError_t setup_paged_attn();
cudaError_t launch_paged_tc(const PagedArgs& a, bool e4m3, int num_sms, PagedEncode encode, cudaStream_t stream);
cudaError_t setup_paged_tc();
// What the call will take by the one and the other, in us and roughly, from the lengths that the host knows: every sequence as long
// as its table, rows spread evenly.  Fitted to 115 calls (94 drawn at random over all sizes): taking the smaller estimate costs
// 1.4 % over the better kernel each time on average, borders on the query rows alone cost 8.7 %.
float paged_attn_us(const PagedArgs& a, bool e4m3, int query_rows, int num_sms);
float paged_tc_us(const PagedArgs& a, bool e4m3, int num_sms);

// Query tiles of a call at most, whatever its lengths: none is without a row, and only the last of a sequence's text tokens (of its
// summaries) holds fewer than tokens_per_tile.
inline int64_t paged_most_tiles(const PagedArgs& a)
{
    const int64_t most = (int64_t)a.B * a.rows_max, rows = most < a.rows ? most : a.rows;
    const int64_t n = (rows + (int64_t)a.B * (a.m > 0 ? 2 : 1) * (a.tokens_per_tile - 1)) / a.tokens_per_tile;
    return n < rows ? n : rows;
}

#if defined(__CUDACC__)
// ---- rows and pages -------------------------------------------------------------------------------------------------
// (Lengths, tables and rows are read past L1: a kernel here may start while the one before the one in front of it still reads,
// after which L1 may keep a line that the one in front rewrites.)
// Sequence b's lengths, checked: false for what are no lengths (nothing of such a sequence is touched).
__device__ __forceinline__ bool paged_seq(const PagedArgs& a, int b, int row0, int r1, int first, int& n)
{
    n = r1 - row0;
    if (!paged_lengths_ok(a, row0, r1, first) || (b == 0 && row0 != 0)) {
        atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_ROWS);
        n = 0;
        return false;
    }
    return true;
}

// The page of row x of a sequence's text (summaries), or -1 (entry -1: given back) or -2 (no page of the pool).
__device__ __forceinline__ int paged_page(const PagedArgs& a, int b, bool summ, int x)
{
    const int col = x >> a.page_shift, cols = summ ? a.summ_cols : a.text_cols;
    if (col >= cols) return -2;
    return paged_entry(a, __ldcg((summ ? a.summ_table : a.text_table) + (int64_t)b * cols + col));
}

// ---- query tiles ------------------------------------------------------------------------------------------------------
// A sequence's rows of the call: how many (0: none for this kernel), text tokens before and among them, tiles of text, of summaries.
// kMix: a run that fits into a tile is one, text tokens and summaries together.
struct PagedRun { int n, t0, nt, tt, ts; };
template <bool kMix>
__device__ __forceinline__ PagedRun paged_run(const PagedArgs& a, int b, int row0, int r1, int first)
{
    PagedRun r{};
    paged_seq(a, b, row0, r1, first, r.n);
    if (r.n < a.rows_min || r.n > a.rows_max) r.n = 0;
    if (r.n > 0) {
        r.t0 = paged_texts(a, first);
        r.nt = paged_texts(a, first + r.n) - r.t0;
        r.tt = a.by_tile(r.nt + a.tokens_per_tile - 1);
        r.ts = a.by_tile(r.n - r.nt + a.tokens_per_tile - 1);
        if (kMix && r.n <= a.tokens_per_tile) { r.tt = 1; r.ts = 0; }
    }
    return r;
}

// Tile `item` of the call, counted through the sequences (text tiles of a sequence before its summary tiles), for the whole block.
// The first warp looks for it, 32 sequences at a time, these in descending order of what their last row sees (the others would only
// compete with it for shuffles and shared memory), and leaves it in `found`.  kMany: before that the whole block counts the tiles of
// 32 sequences at a time, up to 1,024 sequences with all loads in flight.  (256 and 1,024 tokens over 100 rows each, 32/8 heads: 73 and
// 627 us without it, 55 and 225 with it; but its mere code costs a call of one token 0.4 us of 7.8, and one of 64 0.5 of 13.5.)
struct PagedFound { PagedTile tile; int order[32], keys[32]; };
template <bool kMix, bool kMany, int kThreads>
__device__ __forceinline__ PagedTile paged_tile(const PagedArgs& a, int item, PagedFound& found)
{
    int base0 = 0;
    if (kMany && a.B > 32) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        constexpr int kWarps = kThreads / 32, kAhead = 32 / kWarps;
        bool here = false;
        for (int at = 0; at < a.B && !here; at += kThreads * kAhead) {
            int rows0[kAhead], rows1[kAhead], firsts[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int b = at + u * kThreads + (int)threadIdx.x;
                rows0[u] = rows1[u] = firsts[u] = 0;
                if (b < a.B) { rows0[u] = __ldcg(a.cu + b); rows1[u] = __ldcg(a.cu + b + 1); firsts[u] = __ldcg(a.cached + b); }
            }
            if (at > 0) __syncthreads();                       // (the counts before have been read)
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                int tiles = 0;
                if (at + u * kThreads < a.B) {
                    const PagedRun r = paged_run<kMix>(a, at + u * kThreads + (int)threadIdx.x, rows0[u], rows1[u], firsts[u]);
                    tiles = (int)__reduce_add_sync(0xffffffffu, (unsigned)(r.tt + r.ts));
                }
                if (lane == 0) found.keys[u * kWarps + warp] = tiles;
            }
            __syncthreads();
            const int tiles = lane < kWarps * kAhead ? found.keys[lane] : 0;
            int sum = tiles;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += up;
            }
            const unsigned past = __ballot_sync(0xffffffffu, sum > item);
            here = past != 0;
            const int src = here ? __ffs(past) - 1 : 31;
            base0 = at + src * 32;
            item -= __shfl_sync(0xffffffffu, here ? sum - tiles : sum, src);
        }
        __syncthreads();                                       // (before `keys` serves for the order)
        if (!here) base0 = a.B;
    }
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x, per = a.tokens_per_tile;
        PagedTile t{-1, false, false, 0, 0, 0, 0};
        for (int base = base0; base < a.B; base += 32) {
            int row0 = 0, first = 0;
            PagedRun r{};
            if (base + lane < a.B) {
                row0 = __ldcg(a.cu + base + lane);
                first = __ldcg(a.cached + base + lane);
                r = paged_run<kMix>(a, base + lane, row0, __ldcg(a.cu + base + lane + 1), first);
            }
            int n = r.n, t0 = r.t0, nt = r.nt, tt = r.tt, ts = r.ts;
            int seq = base + lane;
            if (a.B > 1) {
                // a lane's place among the 32, by the keys in view (ties by lane), then everything to its place
                const bool summ = n > 0 && nt == 0;
                const PagedView w = paged_view(a, summ, summ ? first + n - t0 - 1 : t0 + max(nt - 1, 0));
                const int keys = n > 0 ? w.t_hi - w.t_lo + w.s_hi - w.s_lo : -1;
                found.keys[lane] = keys;
                __syncwarp();
                int place = 0;
#pragma unroll
                for (int o = 0; o < 32; o += 4) {
                    const int4 k = *reinterpret_cast<const int4*>(found.keys + o);
                    place += (k.x > keys || (k.x == keys && o < lane)) + (k.y > keys || (k.y == keys && o + 1 < lane)) +
                             (k.z > keys || (k.z == keys && o + 2 < lane)) + (k.w > keys || (k.w == keys && o + 3 < lane));
                }
                found.order[place] = lane;
                __syncwarp();
                const int from = found.order[lane];
                seq = base + from;
                row0 = __shfl_sync(0xffffffffu, row0, from); n = __shfl_sync(0xffffffffu, n, from); first = __shfl_sync(0xffffffffu, first, from);
                t0 = __shfl_sync(0xffffffffu, t0, from); nt = __shfl_sync(0xffffffffu, nt, from); tt = __shfl_sync(0xffffffffu, tt, from); ts = __shfl_sync(0xffffffffu, ts, from);
            }
            int sum = tt + ts;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += up;
            }
            const int total = __shfl_sync(0xffffffffu, sum, 31);
            if (item < total) {
                const int src = __ffs(__ballot_sync(0xffffffffu, sum > item)) - 1;
                if (lane == src) {
                    int i = item - (sum - tt - ts);
                    t.b = seq;
                    t.row0 = row0;
                    t.first = first;
                    t.mixed = kMix && n <= per;
                    t.summ = i >= tt;
                    if (t.summ) i -= tt;
                    const int have = t.mixed ? n : t.summ ? n - nt : nt;
                    t.x0 = t.mixed ? first : (t.summ ? first - t0 : t0) + i * per;
                    t.n = min(per, have - i * per);
                    found.tile = t;
                }
                item = -1;
                break;
            }
            item -= total;
        }
        if (item >= 0 && lane == 0) found.tile = t;
    }
    __syncthreads();
    return found.tile;
}

// ---- e4m3 rows ------------------------------------------------------------------------------------------------------------
// 2^(e - 127); 255: NaN
__device__ __forceinline__ float e8m0_scale(uint32_t e)
{
    return __uint_as_float(e == 255u ? 0x7fc00000u : e == 0u ? 0x00400000u : e << 23);
}
// Four e4m3 values as f16, exact: bytes 0, 1 and bytes 2, 3
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
// fp32 -> f16x2 (lo in the low half)
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// 2^(e - 127) for the products: 255, whose row is all zeros, as an infinity, which makes NaN of them
__device__ __forceinline__ float e8m0_factor(uint32_t e) { return __uint_as_float(max(e << 23, 0x00400000u)); }
// Two e4m3 values (low byte first) as fp32
__device__ __forceinline__ float2 e4m3x2_to_f32(uint32_t two)
{
    float2 f;
    asm("{\n\t.reg .b32 h;\n\t.reg .b16 w, lo, hi;\n\t"
        "cvt.u16.u32 w, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 h, w;\n\t"
        "mov.b32 {lo, hi}, h;\n\t"
        "cvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}"
        : "=f"(f.x), "=f"(f.y) : "r"(two));
    return f;
}
#endif

}  // namespace ksa
