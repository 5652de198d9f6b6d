// Attention of a run of new rows over the paged KV cache: tiles of up to 8 or 16 query rows.
//
// A query tile is up to 8 N rows (N = 1 or 2) of one sequence and KV head, (token, query head of the group) each, so that a
// token's whole group reads every key once; what the tile sees is one range of summaries and one of text (Eq. 3; a summary:
// its own chunk).  With so few rows the work is bound by the bytes of K and V.  The key tiles of the two ranges are split
// over the CTAs of a cluster and over each CTA's warps.  A warp has its own ring of stages in shared memory, filled by TMA, a
// box for each run of 16 rows (the pages' least size) by a lane of its own, and waits for no other warp until the end.
// Partial results meet in shared memory, those of the CTAs in distributed shared memory, each CTA of the cluster summing up its
// share of the output's elements: a call is one launch, needs no workspace and adds in a fixed order.
//
// The keys are the M rows of the products, S^T = K Q^T and O^T += V^T P^T with mma.sync m16n8k16, so that 8 query rows take
// half the products, half the registers of O and half of its rescaling that they would as 16 rows of M; P^T gets from the
// first product's layout to the second's by movmatrix.  Running maximum and sum in fp32.
//
// bf16 rows: P rounded to bf16.  e4m3 rows become f16 in registers on their way into the products, one conversion for two
// values (products of e4m3 take e4m3 on both sides, and Q and P would keep four bits of theirs).  So Q becomes f16 too, its
// row scaled by a power of two, and the scale of a key multiplies its scores.  The scale of a value row goes into the
// exponent, u = 2^(score + e - 127 - reference) with the reference maximum taken over these sums: u is at most 2^8 and what f16
// rounds off or loses is relative to the largest that the row has met, whatever the scales are.  The softmax's sum has a
// reference of its own, over the scores: from u it would be u 2^(127 - e), and since the scales span 2^-110 .. 2^120, either
// may be beyond fp32 where the other is about one.  (An exponential and a
// maximum more a score, some constants fewer: 32 tokens over 147,451 rows each 110.9 and 110.1 us, timed in turn.)
// A key's 16 bytes hold four values for each of four lanes; which of the 16 columns a product calls its k-th
// does not matter as long as Q agrees, so lane t takes columns 4 t .. 4 t + 3 as they stand.  Of V, ldmatrix.trans hands a lane
// two neighbouring columns of two keys, which become rows r and r + 8 of a product.
//
// Measured: 32 tokens, each over 147,451 rows, 32/4 heads of 128: bf16 180 us = 6,300 GB/s (a copy: 6,465), e4m3 110 us = 5,190 GB/s,
// the conversions, the products and HBM about level; one token over 9,219 rows, 32/8 heads, bf16: 8.0 us.
#include <cuda_bf16.h>

#include <algorithm>

#include "ksa_launch.h"
#include "ksa_paged.h"
#include "ksa_ptx.cuh"
#include "ksa_wait.cuh"

namespace ksa {

constexpr int kPgRun = 16;                      // rows of a box: the pages' least size
constexpr int kPgMaxSplit = 8;                  // CTAs of a cluster: the portable size

struct PgMaps { CUtensorMap k, v; };

template <int D, bool E4M3, int N>
struct PgCfg {
    static constexpr int kSubs = E4M3 ? 2 : 1;                  // runs in a warp's tile
    static constexpr int kKeys = kPgRun * kSubs;
    static constexpr int kWarps = 4, kThreads = 32 * kWarps;
    static constexpr int kTile = kWarps * kKeys;                // keys of a CTA's tile
    static constexpr int kRows = 8 * N;                         // of the query tile
    static constexpr int kRowB = E4M3 ? D : D * 2;              // bytes of a cached row
    static constexpr int kPanelB = kRowB < 128 ? kRowB : 128;   // a box's width: 128 bytes at most with a swizzle
    static constexpr int kPanels = kRowB / kPanelB;
    static constexpr int kRunB = kPgRun * kRowB;                // of K or of V: its panels, 16 rows each
    static constexpr int kVOff = kSubs * kRunB;
    static constexpr int kStageB = 2 * kVOff;                   // K, V (multiples of 1,024 bytes, which the swizzles repeat after)
    static constexpr int kScaleB = E4M3 ? 2 * kKeys : 0;        // a stage's scale bytes: run by run 16 of K, 16 of V
    static constexpr int kTxBytes = 2 * kVOff;
    static constexpr int kStages = 3;
    static constexpr int kRingB = kStages * kStageB;            // of a warp
    // log2 units.  The reference maximum moves when a score outgrows it by this
    static constexpr float kRescale = 8.0f;
    // bf16: what P stands below 2^(score - reference), so that O, a sum of P V, is within fp32 for V up to 2^128 and down to 2^-90
    static constexpr float kLow = E4M3 ? 0.0f : 30.0f, kUnit = E4M3 ? 1.0f : 0x1p30f;
    static constexpr int kLd = D + 4;                           // floats from one row of partial results to the next
    static constexpr int kMl = E4M3 ? 4 : 2;                    // floats of a row beside O: maximum, sum; e4m3: the sum's own maximum
    static constexpr int kMergeB = kWarps * kRows * (kLd + kMl) * 4;    // the warps' results, over the ring
    // what the cluster's other CTAs push: memory of its own, this CTA may still be at work
    static constexpr int kPushOff = kWarps * kRingB > kMergeB ? kWarps * kRingB : kMergeB;
    static constexpr int kPushO = (kRows * (D / 4) + kPgMaxSplit) * 16, kPushMl = kPgMaxSplit * kRows * kMl * 4;
    static constexpr int kScaleOff = kPushOff + kPushO + kPushMl;       // [warps][stages]
    static constexpr int kBarOff = kScaleOff + kWarps * kStages * kScaleB;
    static constexpr int kSmemBytes = kBarOff + 8 * kWarps * kStages + 16 + 1024;       // + slack for 1024-byte alignment
    // 16-byte vector c of row r of a run, as the boxes' swizzles place them
    __device__ static __forceinline__ uint32_t at(int r, int c)
    {
        return (uint32_t)((c >> 3) * (kPgRun * 128) + r * kPanelB + (((c & 7) ^ (kPanelB == 64 ? (r >> 1) & 3 : r & 7)) << 4));
    }
};

__device__ __forceinline__ void pg_ldsm(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void pg_ldsm_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t pg_transpose(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void pg_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2])
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void pg_mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2])
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t pg_ld_u8(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}

template <int D, bool E4M3, int N, bool kMany>
__global__ void __launch_bounds__(PgCfg<D, E4M3, N>::kThreads) ksa_paged_attn_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PgMaps maps)
{
    using Cfg = PgCfg<D, E4M3, N>;
    constexpr int kStages = Cfg::kStages, kSubs = Cfg::kSubs, kKeys = Cfg::kKeys, kTile = Cfg::kTile, kWarps = Cfg::kWarps, kThreads = Cfg::kThreads;
    extern __shared__ uint8_t pgsm_raw[];
    uint8_t* pgsm = pgsm_raw + (-ptx::smem_u32(pgsm_raw) & 1023u);
    const uint32_t sbase = ptx::smem_u32(pgsm);
    const uint32_t bars = sbase + Cfg::kBarOff, abort_addr = bars + 8 * kWarps * kStages;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWarps * kStages; ++i) ptx::mbar_init(bars + 8 * i, 1);
        st_shared_u32(abort_addr, 0u);
        st_shared_u32(abort_addr + 4, 0u);                     // never raised: lets the last waits run while aborting
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&maps.k);
        ptx::prefetch_tensormap(&maps.v);
    }
    __syncthreads();
    if (a.nsplit > 1) ptx::cluster_arrive();                   // (waited for before the first access to another CTA's memory)
    if (a.beside == 0) ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    if (a.beside == 1) ptx::pdl_launch_dependents();           // the kernel behind does not wait for this one, but for those before
    const int unit = a.by_split((int)blockIdx.x), split = (int)blockIdx.x - unit * a.nsplit;
    const int item = a.by_heads(unit), hkb = unit - item * a.Hkv * a.head_blocks, hk = a.by_group(hkb), hb = hkb - hk * a.head_blocks;
    __shared__ __align__(16) PagedFound found;
    const PagedTile t = paged_tile<false, kMany, Cfg::kThreads>(a, item, found);
    if (t.b < 0) return;                                       // (the whole cluster)
    const int l4 = lane >> 2, c2 = (lane & 3) * 2;             // fragment row and column pair
    // the tile's rows: (token, head), heads `head0 ..` of the group
    const int head0 = hk * a.G + hb * Cfg::kRows, heads = min(Cfg::kRows, a.G - hb * Cfg::kRows), nrow = t.n * heads;
    // what anything in the tile sees; rows that all of it sees: a warp's keys within them need no mask
    const PagedView see = paged_tile_view(a, t), first = paged_view(a, t.summ, t.x0), last = paged_view(a, t.summ, t.x0 + t.n - 1);
    const int s_t0 = see.s_lo / kTile, s_tiles = see.s_hi > see.s_lo ? (see.s_hi + kTile - 1) / kTile - s_t0 : 0;
    const int t_t0 = see.t_lo / kTile, tiles = s_tiles + (see.t_hi + kTile - 1) / kTile - t_t0;
    // the cluster's CTAs that take part: a CTA without two key tiles of its own leaves (the others' barriers do not count it)
    const int parts = min(a.nsplit, max(1, tiles >> 1));
    if (split >= parts) return;
    const int per = (tiles + parts - 1) / parts;
    const int my0 = min(tiles, split * per), my1 = min(tiles, my0 + per);

    // First row of the warp's tile j in its stream.
    auto tile_at = [&](int j, bool& summ) { summ = j < s_tiles; return (summ ? s_t0 + j : t_t0 + j - s_tiles) * kTile + warp * kKeys; };
    // Q, as it comes: columns 4 t .. 4 t + 3 of 16 (bf16 rows: 2 t, 2 t + 1 and 8 + 2 t, 9 + 2 t); on its way beside the first keys
    uint2 qw[N][D / 16];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int r = min(n * 8 + l4, nrow - 1);
        const uint16_t* q = a.q + paged_row(a, t, t.x0 + r / heads) * a.q_st + (head0 + r % heads) * a.q_sh;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            if constexpr (E4M3) qw[n][kk] = __ldcg(reinterpret_cast<const uint2*>(q + kk * 16 + c2 * 2));
            else qw[n][kk] = make_uint2(__ldcg(reinterpret_cast<const uint32_t*>(q + kk * 16 + c2)), __ldcg(reinterpret_cast<const uint32_t*>(q + kk * 16 + 8 + c2)));
        }
    }
    // Lane u < kSubs brings the tile's run u.  Its page-table entry is fetched a tile ahead of its use; -3: nobody sees the rows.
    auto find_entry = [&](int j) {
        bool summ;
        const int x = tile_at(j, summ) + kPgRun * lane, col = x >> a.page_shift, cols = summ ? a.summ_cols : a.text_cols;
        if (lane >= kSubs || j >= my1 || x >= (summ ? see.s_hi : see.t_hi) || x + kPgRun <= (summ ? see.s_lo : see.t_lo)) return -3;
        return col < cols ? __ldcg((summ ? a.summ_table : a.text_table) + (int64_t)t.b * cols + col) : -2;
    };
    const uint32_t ring = sbase + warp * Cfg::kRingB, full = bars + 8 * warp * kStages, scales = sbase + Cfg::kScaleOff + warp * kStages * Cfg::kScaleB;
    auto load_tile = [&](int j, int stage, int entry) {
        if (lane == 0) ptx::mbar_arrive_expect_tx(full + 8 * stage, Cfg::kTxBytes);
        bool summ;
        const int row0 = tile_at(j, summ) & ((1 << a.page_shift) - 1);
        int page = paged_entry(a, entry);
        if (page < 0) {
            if (lane < kSubs && entry != -3) atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_PAGE);
            page = a.num_pages;                                // outside the pool: a box of zeros
        }
        int box_page = page;
        if constexpr (kSubs == 2) {                            // one box for both runs: the page of the one that is seen
            const int other = __shfl_sync(0xffffffffu, page, 1);
            if (a.box_rows == 2 * kPgRun && page == a.num_pages) box_page = other;
        }
        __syncwarp();
        if (lane < kSubs && (lane == 0 || a.box_rows == kPgRun)) {
            const uint32_t sk = ring + stage * Cfg::kStageB + lane * Cfg::kRunB, bar = full + 8 * stage;
            const int row = row0 + lane * kPgRun & ((1 << a.page_shift) - 1);
#pragma unroll
            for (int p = 0; p < Cfg::kPanels; ++p) {
                ptx::tma_load_4d(sk + p * (kPgRun * 128), &maps.k, bar, p * (Cfg::kPanelB / (E4M3 ? 1 : 2)), row, hk, box_page);
                ptx::tma_load_4d(sk + Cfg::kVOff + p * (kPgRun * 128), &maps.v, bar, p * (Cfg::kPanelB / (E4M3 ? 1 : 2)), row, hk, box_page);
            }
        }
        if constexpr (E4M3) {                                  // lanes 0, 1: the runs' scale bytes of K, lanes 2, 3: of V
            const int u = lane & 1, from = __shfl_sync(0xffffffffu, page, u);
            if (lane < 4 && from < a.num_pages) {
                const int64_t at = (((int64_t)from * a.Hkv + hk) << a.page_shift) + (row0 + u * kPgRun & ((1 << a.page_shift) - 1));
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(scales + stage * Cfg::kScaleB + u * 32 + (lane >> 1) * 16), "l"((lane < 2 ? a.ke : a.ve) + at) : "memory");
            }
        }
    };
    int entry;
    {
        int early[kStages - 1];
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) early[s] = find_entry(my0 + s);
        entry = find_entry(my0 + kStages - 1);
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) {
            if (my0 + s < my1) load_tile(my0 + s, s, early[s]);
            if constexpr (E4M3) asm volatile("cp.async.commit_group;" ::: "memory");
        }
    }
    // Q^T fragments (B operand, D x 8 N); rows past the tile's are zero
    uint32_t qb[D / 16][N][2];
    float qf[N][2];                                            // e4m3: what the scores of rows 8 n + c2, + 1 are to be multiplied with
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const bool ok = n * 8 + l4 < nrow;
        if constexpr (E4M3) {
            // As f16, the row scaled by a power of two to a largest value of 2^8 .. 2^9: exact down to 2^-22 of that, and off by 2^-33 of
            // it below
            uint32_t top = 0;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) top = __vmaxu2(top, __vmaxu2(qw[n][kk].x & 0x7fff7fffu, qw[n][kk].y & 0x7fff7fffu));
            top = max(top >> 16, top & 0xffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = min(max((int)(top >> 7) - 8, 1), 253);                  // the scale is 2^(127 - e), its inverse 2^(e - 127)
            const float f = __uint_as_float((uint32_t)(254 - e) << 23);
            auto two = [&](uint32_t x) { const uint32_t h = pack_f16x2(__uint_as_float(x << 16) * f, __uint_as_float(x & 0xffff0000u) * f); return ok ? h : 0u; };
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) { qb[kk][n][0] = two(qw[n][kk].x); qb[kk][n][1] = two(qw[n][kk].y); }
            const float back = __uint_as_float((uint32_t)e << 23);             // (lane 4 i holds row i)
            qf[n][0] = __shfl_sync(0xffffffffu, back, c2 * 4);
            qf[n][1] = __shfl_sync(0xffffffffu, back, c2 * 4 + 4);
        } else {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) { qb[kk][n][0] = ok ? qw[n][kk].x : 0u; qb[kk][n][1] = ok ? qw[n][kk].y : 0u; }
        }
    }
    float o[D / 16][N][4];
    float m[N][2], l[N][2], ml[N][2];                          // of query rows 8 n + c2, + 1; e4m3: ml is the reference of the sum
#pragma unroll
    for (int n = 0; n < N; ++n) {
        m[n][0] = m[n][1] = ml[n][0] = ml[n][1] = -INFINITY; l[n][0] = l[n][1] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) { o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f; }
    }
    const int mi = lane >> 3, r8 = lane & 7;
    int stage = 0;
    uint32_t phase = 0;
    for (int j = my0; j < my1; ++j) {
        __syncwarp();                                          // the tile before has been read by every lane
        if (j + kStages - 1 < my1) load_tile(j + kStages - 1, stage == 0 ? kStages - 1 : stage - 1, entry);
        if constexpr (E4M3) asm volatile("cp.async.commit_group;" ::: "memory");
        entry = find_entry(j + kStages);
        if constexpr (E4M3) asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        const bool ok = bounded_wait(full + 8 * stage, phase, abort_addr, a.status, kStatusWaitKvFull);
        if (!__all_sync(0xffffffffu, ok)) {                    // given up: no copy is left in flight behind
            for (int i = j, st = stage; i < min(j + kStages, my1); ++i) {
                bounded_wait(full + 8 * st, phase, abort_addr + 4, a.status, kStatusWaitKvFull);
                if (++st == kStages) { st = 0; phase ^= 1u; }
            }
            break;
        }
        __syncwarp();
        const uint32_t sk = ring + stage * Cfg::kStageB, sv = sk + Cfg::kVOff, sc = scales + stage * Cfg::kScaleB;
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
        bool summ;
        const int x0 = tile_at(j, summ);
        const int lo = summ ? see.s_lo : see.t_lo, hi = summ ? see.s_hi : see.t_hi;
        if (x0 >= hi || x0 + kKeys <= lo) continue;            // nobody sees any of it
        if (x0 < lo || x0 + kKeys > hi) {                      // V of rows that nobody sees: zeros (0 times what stands there may be NaN)
            constexpr int kVec = Cfg::kRowB / 16;
            for (int i = lane; i < kKeys * kVec; i += 32) {
                const int r = i / kVec;
                if (x0 + r < lo || x0 + r >= hi)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sv + (r >> 4) * Cfg::kRunB + Cfg::at(r & 15, i % kVec)), "r"(0u) : "memory");
            }
            ptx::fence_proxy_async();                          // (before the stage is filled again)
            __syncwarp();
        }
        // S^T (16 keys x 8 N query rows, run by run) = K Q^T, in log2 units
        float s[kSubs][N][4], r[kSubs][N][4];                  // e4m3: with the value rows' exponents, and without
#pragma unroll
        for (int u = 0; u < kSubs; ++u) {
#pragma unroll
            for (int n = 0; n < N; ++n) { s[u][n][0] = s[u][n][1] = s[u][n][2] = s[u][n][3] = 0.f; }
            if constexpr (E4M3) {
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk) {          // 32 columns
                    uint32_t kb[4];
                    pg_ldsm(kb, sk + u * Cfg::kRunB + Cfg::at((mi & 1) * 8 + r8, kk * 2 + (mi >> 1)));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t a0, a1, a2, a3;
                        e4m3x4_to_f16(kb[2 * i], a0, a2);
                        e4m3x4_to_f16(kb[2 * i + 1], a1, a3);
#pragma unroll
                        for (int n = 0; n < N; ++n) pg_mma_f16(s[u][n], a0, a1, a2, a3, qb[kk * 2 + i][n]);
                    }
                }
                const uint32_t se = sc + u * 32 + l4;
#pragma unroll
                for (int h = 0; h < 2; ++h) {                  // keys l4, l4 + 8
                    const float fk = a.scale_log2 * e8m0_factor(pg_ld_u8(se + 8 * h));
                    const uint32_t e = pg_ld_u8(se + 16 + 8 * h);
                    const float ef = e == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(0x4b000000u | e) - (8388608.f + 127.f);
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            r[u][n][2 * h + c] = s[u][n][2 * h + c] * qf[n][c] * fk;
                            s[u][n][2 * h + c] = r[u][n][2 * h + c] + ef;
                        }
                }
            } else {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    uint32_t kb[4];
                    pg_ldsm(kb, sk + u * Cfg::kRunB + Cfg::at((mi & 1) * 8 + r8, kk * 2 + (mi >> 1)));
#pragma unroll
                    for (int n = 0; n < N; ++n) pg_mma(s[u][n], kb[0], kb[1], kb[2], kb[3], qb[kk][n]);
                }
#pragma unroll
                for (int n = 0; n < N; ++n) { s[u][n][0] *= a.scale_log2; s[u][n][1] *= a.scale_log2; s[u][n][2] *= a.scale_log2; s[u][n][3] *= a.scale_log2; }
            }
        }
        // each row's own range, where the keys hold an end of some row's
        if (x0 < (summ ? last.s_lo : last.t_lo) || x0 + kKeys > (summ ? first.s_hi : first.t_hi)) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const PagedView w = paged_view(a, t.summ, t.x0 + min(n * 8 + c2 + c, nrow - 1) / heads);
                    const int rlo = (summ ? w.s_lo : w.t_lo) - x0 - l4, rhi = (summ ? w.s_hi : w.t_hi) - x0 - l4;
#pragma unroll
                    for (int u = 0; u < kSubs; ++u)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (16 * u + 8 * h < rlo || 16 * u + 8 * h >= rhi) {
                                s[u][n][2 * h + c] = -INFINITY;
                                if constexpr (E4M3) r[u][n][2 * h + c] = -INFINITY;
                            }
                }
        }
        // the reference maximum moves, and O with it, only when some row outgrew its own (eight lanes share a row)
        float mx[N][2], rx[N][2];
        bool grown = false;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                mx[n][c] = fmaxf(s[0][n][c], s[0][n][2 + c]);
#pragma unroll
                for (int u = 1; u < kSubs; ++u) mx[n][c] = ptx::fmax3(mx[n][c], s[u][n][c], s[u][n][2 + c]);
                grown |= mx[n][c] > m[n][c] + Cfg::kRescale;
                if constexpr (E4M3) {
                    rx[n][c] = fmaxf(r[0][n][c], r[0][n][2 + c]);
#pragma unroll
                    for (int u = 1; u < kSubs; ++u) rx[n][c] = ptx::fmax3(rx[n][c], r[u][n][c], r[u][n][2 + c]);
                    grown |= rx[n][c] > ml[n][c] + Cfg::kRescale;
                }
            }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = mx[n][c];
#pragma unroll
                    for (int b = 4; b < 32; b <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, b));
                    const float mn = fmaxf(m[n][c], x), al = (mn == -INFINITY) ? 1.f : ptx::ex2_approx(m[n][c] - mn);
                    m[n][c] = mn;
                    if constexpr (E4M3) {
                        x = rx[n][c];
#pragma unroll
                        for (int b = 4; b < 32; b <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, b));
                        const float rn = fmaxf(ml[n][c], x);
                        l[n][c] *= (rn == -INFINITY) ? 1.f : ptx::ex2_approx(ml[n][c] - rn);
                        ml[n][c] = rn;
                    } else {
                        l[n][c] *= al;
                    }
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) { o[i][n][c] *= al; o[i][n][2 + c] *= al; }
                }
        }
#pragma unroll
        for (int u = 0; u < kSubs; ++u) {
            uint32_t pb[N][2];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const float sub0 = (m[n][0] == -INFINITY) ? 0.f : m[n][0] + Cfg::kLow, sub1 = (m[n][1] == -INFINITY) ? 0.f : m[n][1] + Cfg::kLow;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float p0 = ptx::ex2_approx(s[u][n][2 * h] - sub0), p1 = ptx::ex2_approx(s[u][n][2 * h + 1] - sub1);
                    if constexpr (E4M3) {
                        l[n][0] += ptx::ex2_approx(r[u][n][2 * h] - ((ml[n][0] == -INFINITY) ? 0.f : ml[n][0]));
                        l[n][1] += ptx::ex2_approx(r[u][n][2 * h + 1] - ((ml[n][1] == -INFINITY) ? 0.f : ml[n][1]));
                        pb[n][h] = pg_transpose(pack_f16x2(p0, p1));
                    } else {
                        l[n][0] += p0;
                        l[n][1] += p1;
                        pb[n][h] = pg_transpose(ptx::pack_bf16x2(p0, p1));
                    }
                }
            }
            // O^T += V^T P^T
            if constexpr (E4M3) {                              // rows r, r + 8 of a product: columns 2 r, 2 r + 1 of 16
#pragma unroll
                for (int i2 = 0; i2 < D / 32; ++i2) {
                    uint32_t vb[4];
                    pg_ldsm_t(vb, sv + u * Cfg::kRunB + Cfg::at((mi & 1) * 8 + r8, i2 * 2 + (mi >> 1)));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t a0, a1, a2, a3;
                        e4m3x4_to_f16(__byte_perm(vb[2 * i], 0, 0x3120), a0, a1);
                        e4m3x4_to_f16(__byte_perm(vb[2 * i + 1], 0, 0x3120), a2, a3);
#pragma unroll
                        for (int n = 0; n < N; ++n) pg_mma_f16(o[2 * i2 + i][n], a0, a1, a2, a3, pb[n]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    uint32_t vb[4];
                    pg_ldsm_t(vb, sv + u * Cfg::kRunB + Cfg::at((mi >> 1) * 8 + r8, i * 2 + (mi & 1)));
#pragma unroll
                    for (int n = 0; n < N; ++n) pg_mma(o[i][n], vb[0], vb[1], vb[2], vb[3], pb[n]);
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int b = 4; b < 32; b <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], b);
    if constexpr (E4M3) asm volatile("cp.async.wait_all;" ::: "memory");
    // the warps' results: rows of (maximum, sum; e4m3: the sum's maximum) and of O each
    __syncthreads();
    constexpr int kRows = Cfg::kRows, kLd = Cfg::kLd, kMl = Cfg::kMl;
    float* sm_o = reinterpret_cast<float*>(pgsm);                      // [warps][rows][kLd]
    float* sm_ml = sm_o + kWarps * kRows * kLd;                        // [warps][rows][kMl]
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float* r = sm_o + (warp * kRows + n * 8 + c2 + e) * kLd;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                if constexpr (E4M3) *reinterpret_cast<float2*>(r + i * 16 + 2 * l4) = make_float2(o[i][n][e], o[i][n][2 + e]);
                else { r[i * 16 + l4] = o[i][n][e]; r[i * 16 + 8 + l4] = o[i][n][2 + e]; }
            }
            if (l4 == 0) {
                float* to = sm_ml + (warp * kRows + n * 8 + c2 + e) * kMl;
                *reinterpret_cast<float2*>(to) = make_float2(m[n][e], l[n][e]);
                if constexpr (E4M3) to[2] = ml[n][e];
            }
        }
    __syncthreads();
    // A row's O relative to 2^M, its sum relative to 2^ML (bf16: M and ML are one), of all warps (CTAs) so far: the next ones' added
    struct Row { float M, ML, L; float4 acc; };
    auto reference = [&](const float* x, Row& w) { w.M = fmaxf(w.M, x[0]); if constexpr (E4M3) w.ML = fmaxf(w.ML, x[2]); };
    auto add = [&](const float* x, const float4& v, Row& w) {
        const float f = (x[0] == -INFINITY) ? 0.f : ptx::ex2_approx(x[0] - w.M);
        if constexpr (E4M3) w.L += (x[2] == -INFINITY) ? 0.f : x[1] * ptx::ex2_approx(x[2] - w.ML); else w.L += x[1] * f;
        w.acc.x += v.x * f; w.acc.y += v.y * f; w.acc.z += v.z * f; w.acc.w += v.w * f;
    };
    auto write = [&](int g, int d, const Row& w) {
        // (2^(M - ML) in two halves: it may be past 2^127 where what it multiplies is small)
        const float half = E4M3 ? ptx::ex2_approx(0.5f * (w.M - w.ML)) : 1.f, inv = half / w.L;
        const float4& acc = w.acc;
        const int64_t row = paged_row(a, t, t.x0 + g / heads);
        const int h = head0 + g % heads;
        if (!ksa_in_bounds(row >= 0 && row < a.rows && h < a.Hq, a.status)) return;
        *reinterpret_cast<uint2*>(a.out + row * a.o_st + h * a.o_sh + d) =
            make_uint2(ptx::pack_bf16x2(acc.x * inv * half, acc.y * inv * half), ptx::pack_bf16x2(acc.z * inv * half, acc.w * inv * half));
        if (d == 0) a.lse[(int64_t)h * a.rows + row] = ((E4M3 ? w.ML : w.M) + log2f(w.L * Cfg::kUnit)) * 0.6931471805599453f;
    };
    // Each CTA of the cluster sums up a share of the output's elements (4 columns of a row each), `share` of them: the others
    // write what they have of these into its memory, where the one barrier finds everything.
    const int total = nrow * (D / 4), share = (total + parts - 1) / parts;
    const uint32_t push_o = sbase + Cfg::kPushOff, push_ml = push_o + Cfg::kPushO;       // [parts][share] of 16 bytes, [parts][rows][kMl] floats
    if (parts > 1) ptx::cluster_wait();                        // they have all started
    for (int idx = threadIdx.x; idx < total; idx += kThreads) {
        const int g = idx / (D / 4), d = (idx - g * (D / 4)) * 4;
        Row w{-INFINITY, -INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < kWarps; ++i) reference(sm_ml + (i * kRows + g) * kMl, w);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) add(sm_ml + (i * kRows + g) * kMl, *reinterpret_cast<const float4*>(sm_o + (i * kRows + g) * kLd + d), w);
        if (parts == 1) {
            write(g, d, w);
        } else {
            const int to = idx / share;
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                         ::"r"(ptx::mapa_shared(push_o + (split * share + idx - to * share) * 16, to)), "f"(w.acc.x), "f"(w.acc.y), "f"(w.acc.z), "f"(w.acc.w) : "memory");
            if (d == 0)
                for (int p = 0; p < parts; ++p) {
                    const uint32_t at = ptx::mapa_shared(push_ml + (split * kRows + g) * kMl * 4, p);
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(w.M), "f"(w.L) : "memory");
                    if constexpr (E4M3) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(w.ML) : "memory");
                }
        }
    }
    if (parts > 1) {
        __syncwarp();
        ptx::cluster_arrive();
        ptx::cluster_wait();
        const float4* po = reinterpret_cast<const float4*>(pgsm + Cfg::kPushOff);
        const float* pm = reinterpret_cast<const float*>(pgsm + Cfg::kPushOff + Cfg::kPushO);
        for (int e = threadIdx.x; e < share && split * share + e < total; e += kThreads) {
            const int idx = split * share + e, g = idx / (D / 4), d = (idx - g * (D / 4)) * 4;
            Row w{-INFINITY, -INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
            for (int p = 0; p < parts; ++p) reference(pm + (p * kRows + g) * kMl, w);
#pragma unroll 4
            for (int p = 0; p < parts; ++p) add(pm + (p * kRows + g) * kMl, po[p * share + e], w);
            write(g, d, w);
        }
    }
}

// f(kernel, shared memory, threads) for one of the kernels
template <int D, bool E4M3, int N, class F> static cudaError_t with_kernel(bool many, F f)
{
    using Cfg = PgCfg<D, E4M3, N>;
    return many ? f(ksa_paged_attn_kernel<D, E4M3, N, true>, Cfg::kSmemBytes, Cfg::kThreads) : f(ksa_paged_attn_kernel<D, E4M3, N, false>, Cfg::kSmemBytes, Cfg::kThreads);
}
template <int D, class F> static cudaError_t with_kernel(bool e4m3, int n, bool many, F f)
{
    if (e4m3) return n == 1 ? with_kernel<D, true, 1>(many, f) : with_kernel<D, true, 2>(many, f);
    return n == 1 ? with_kernel<D, false, 1>(many, f) : with_kernel<D, false, 2>(many, f);
}
cudaError_t setup_paged_attn()
{
    auto set = [](auto kernel, int smem, int) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); };
    for (bool many : {false, true})
        for (int n : {1, 2})
            for (bool e4m3 : {false, true})
                for (const cudaError_t e : {with_kernel<128>(e4m3, n, many, set), with_kernel<64>(e4m3, n, many, set)})
                    if (e != cudaSuccess) return e;
    return cudaSuccess;
}

// CTAs of one cluster for a call of `units` query tiles at most, as far as there are key tiles to split: two up to ten CTAs an SM in
// the grid, more up to five (two are resident).  128 units of 17,300 rows each, e4m3 (1, 2, 4, 8 CTAs a unit): 186, 94, 102,
// 117 us; 116 units of 700 to 17,400 rows: 199, 103, 59, 65 us; 8 units of 2,000 rows, bf16: 29, 17, 10.7, 7.8 us; up to 384 units,
// 16 sequences of 6 drafted rows, e4m3 (1, 2): 70, 57 us.
static int paged_splits(int64_t units, int64_t key_tiles, int num_sms)
{
    int n = 1;
    while (n < kPgMaxSplit && units * n * 2 <= (n == 1 ? 10 : 5) * num_sms && key_tiles >= 4 * n) n *= 2;       // (a CTA takes two tiles at least)
    return n;
}

bool encode_pages(PagedEncode encode, CUtensorMap* map, void* base, const PagedArgs& a, bool e4m3, int box_bytes, int box_rows, CUtensorMapSwizzle swizzle)
{
    const cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)1 << a.page_shift, (cuuint64_t)a.Hkv, (cuuint64_t)a.num_pages};
    auto stride = [](int64_t st) { return (cuuint64_t)(st > 0 ? st : 16); };            // (0: a dimension of one)
    const cuuint64_t strides[3] = {stride(a.row_st), stride(a.head_st), stride(a.page_st)};
    const cuuint32_t box[4] = {(cuuint32_t)(e4m3 ? box_bytes : box_bytes / 2), (cuuint32_t)box_rows, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return encode(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Some 6 us, then the key rows that all query tiles walk, 30,000 (e4m3) or 16,000 (bf16) a us on 148 SMs at head_dim 128, and the walk
// of one on the CTAs of a cluster
float paged_attn_us(const PagedArgs& a, bool e4m3, int query_rows, int num_sms)
{
    const int rows = query_rows <= 8 ? 8 : 16, tokens = std::max(1, rows / a.G), blocks = (a.G + rows - 1) / rows;
    const int64_t text = std::min((int64_t)a.text_cols << a.page_shift, ((int64_t)a.C + 2) * a.kk + tokens);
    const float keys = (float)(text + (a.m > 0 ? (int64_t)a.summ_cols << a.page_shift : 0));
    const float tiles = (float)std::max((a.rows + tokens - 1) / tokens, a.B) * (float)(a.Hkv * blocks);
    return 6.0f + tiles * keys / ((e4m3 ? 203.0f : 108.0f) * (float)num_sms * (a.D == 128 ? 1.0f : 1.5f)) + keys / 700.0f;
}

cudaError_t launch_paged_attn(const PagedArgs& args, bool e4m3, int query_rows, int num_sms, PagedEncode encode, cudaStream_t stream)
{
    PagedArgs a = args;
    const int n = query_rows <= 8 ? 1 : 2;
    a.tokens_per_tile = std::max(1, 8 * n / a.G);
    a.head_blocks = (a.G + 8 * n - 1) / (8 * n);
    a.by_tile = PagedDiv::by(a.tokens_per_tile);
    const int64_t units = paged_most_tiles(a) * a.Hkv * a.head_blocks;
    const int64_t rows = ((int64_t)a.text_cols + (a.m > 0 ? a.summ_cols : 0)) << a.page_shift;      // of a sequence, at most
    a.nsplit = paged_splits(units, rows / (e4m3 ? 128 : 64), num_sms);
    a.by_split = PagedDiv::by(a.nsplit);
    a.by_heads = PagedDiv::by(a.Hkv * a.head_blocks); a.by_group = PagedDiv::by(a.head_blocks);
    // (a box of the warp's whole tile where a page holds it: every box costs the warp that asks for it some 50 cycles)
    a.box_rows = e4m3 && a.page_shift > 4 ? 2 * kPgRun : kPgRun;
    const int panel = a.D * (e4m3 ? 1 : 2) < 128 ? 64 : 128;
    const CUtensorMapSwizzle swizzle = panel == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
    PgMaps maps;
    if (!encode_pages(encode, &maps.k, a.kp, a, e4m3, panel, a.box_rows, swizzle) || !encode_pages(encode, &maps.v, a.vp, a, e4m3, panel, a.box_rows, swizzle))
        return cudaErrorInvalidValue;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.nsplit; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(units * a.nsplit)); cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = 2;
    auto go = [&](auto kernel, int smem, int threads) {
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = (size_t)smem;
        return cudaLaunchKernelEx(&cfg, kernel, a, maps);
    };
    const bool many = a.B > 64;                                // (see paged_tile)
    return a.D == 128 ? with_kernel<128>(e4m3, n, many, go) : with_kernel<64>(e4m3, n, many, go);
}

}  // namespace ksa
