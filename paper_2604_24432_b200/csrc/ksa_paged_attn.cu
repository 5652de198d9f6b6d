// Attention of a run of new rows over the paged KV cache: tiles of up to 16 query rows.
//
// A query tile is up to 16 rows of one sequence and KV head, (token, query head of the group) each, so that a token's whole
// group reads every key once; what the tile sees is one range of summaries and one of text (Eq. 3; a summary: its own chunk).
// With so few rows the work is bound by the bytes of K and V.  The 64-row key tiles of the two ranges are split over the
// CTAs of a cluster; a CTA streams its share through a ring of cp.async stages in (swizzled) shared memory, page by page;
// its four warps take 16 keys of each tile: S = Q K^T and O += P V with mma.sync m16n8k16, running maximum and sum of the
// softmax in fp32.  Partial results meet in distributed shared memory: each CTA of the cluster sums up its share of the
// output's elements, so a call is one launch, needs no workspace and adds in a fixed order.
//
// e4m3 rows are taken to bf16 in registers on their way into the products: the scale of a key multiplies its
// scores, that of a value row the probability before it is rounded to bf16.  A key's 16 bytes hold four values for each of four
// lanes; which of the 16 columns a product calls its k-th does not matter as long as Q agrees, so lane t takes
// columns 4 t .. 4 t + 3, as they stand, and loads Q the same way.  Of V, ldmatrix.trans hands a lane two neighbouring
// columns of two keys; they go to two products, one of the even columns and one of the odd ones.
#include <cuda_bf16.h>

#include "ksa_launch.h"
#include "ksa_paged.h"
#include "ksa_ptx.cuh"

namespace ksa {

constexpr int kPgTile = 64;         // cache rows per shared-memory tile
constexpr int kPgThreads = 128;
constexpr int kPgMaxSplit = 8;      // the portable cluster size

template <int D, bool E4M3>
struct PgCfg {
    static constexpr int kRowB = E4M3 ? D : D * 2;              // bytes of a row
    static constexpr int kVec = kRowB / 16;
    static constexpr int kTileB = kPgTile * kRowB;
    static constexpr int kScaleB = E4M3 ? 2 * kPgTile : 0;      // scale bytes of K, then V
    static constexpr int kStageB = 2 * kTileB + kScaleB;
    static constexpr int kStages = E4M3 ? 4 : 3;
    static constexpr int kRingB = kStages * kStageB;
    static constexpr int kMergeB = 4 * 16 * D * 4 + 4 * 16 * 2 * 4 + 16 * D * 4 + 16 * 2 * 4;
    static constexpr int kSmemBytes = kRingB > kMergeB ? kRingB : kMergeB;
};

__device__ __forceinline__ void pg_cp16(uint32_t dst, const void* src, bool valid)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void pg_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void pg_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
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
__device__ __forceinline__ void pg_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two e4m3 values -> bf16x2
__device__ __forceinline__ uint32_t pg_two(uint32_t y)
{
    const float2 f = e4m3x2_to_f32(y & 0xffffu);
    return ptx::pack_bf16x2(f.x, f.y);
}
__device__ __forceinline__ uint32_t pg_ld_u32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ float2 pg_ld_cluster2(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
    return v;
}
__device__ __forceinline__ float4 pg_ld_cluster4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(kPgThreads) ksa_paged_attn_kernel(const __grid_constant__ PagedArgs a)
{
    using Cfg = PgCfg<D, E4M3>;
    constexpr int kStages = Cfg::kStages;
    extern __shared__ __align__(128) uint8_t pgsm[];
    const uint32_t sbase = ptx::smem_u32(pgsm);
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int split = (int)blockIdx.x % a.nsplit, unit = (int)blockIdx.x / a.nsplit;
    const int hb = unit % a.head_blocks, hk = unit / a.head_blocks % a.Hkv;
    const PagedTile t = paged_tile(a, unit / a.head_blocks / a.Hkv);
    if (t.b < 0) return;                                       // (the whole cluster)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g0 = lane >> 2, c2 = (lane & 3) * 2;             // fragment row and column pair
    // the tile's rows: (token, head), heads `head0 ..` of the group
    const int head0 = hk * a.G + hb * 16, heads = min(16, a.G - hb * 16), nrow = t.n * heads;
    const PagedView see = paged_tile_view(a, t);
    const int s_t0 = see.s_lo / kPgTile, s_tiles = see.s_hi > see.s_lo ? (see.s_hi + kPgTile - 1) / kPgTile - s_t0 : 0;
    const int t_t0 = see.t_lo / kPgTile, tiles = s_tiles + (see.t_hi + kPgTile - 1) / kPgTile - t_t0;
    const int per = (tiles + a.nsplit - 1) / a.nsplit;
    const int my0 = min(tiles, split * per), my1 = min(tiles, my0 + per);

    // Q fragments (A operand, 16 x D); rows past the tile's are zero
    uint32_t qa[D / 16][4];
    PagedView v0 = see, v1 = see;                              // what fragment rows g0 and g0 + 8 see
    {
        const int r0 = min(g0, nrow - 1), r1 = min(g0 + 8, nrow - 1);
        const int x0 = t.x0 + r0 / heads, x1 = t.x0 + r1 / heads;
        v0 = paged_view(a, t.summ, x0);
        v1 = paged_view(a, t.summ, x1);
        const uint16_t* q0 = a.q + paged_row(a, t, x0) * a.q_st + (head0 + r0 % heads) * a.q_sh;
        const uint16_t* q1 = a.q + paged_row(a, t, x1) * a.q_st + (head0 + r1 % heads) * a.q_sh;
        const bool ok0 = g0 < nrow, ok1 = g0 + 8 < nrow;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            if constexpr (E4M3) {
                const uint2 w0 = __ldcg(reinterpret_cast<const uint2*>(q0 + kk * 16 + c2 * 2)), w1 = __ldcg(reinterpret_cast<const uint2*>(q1 + kk * 16 + c2 * 2));
                qa[kk][0] = ok0 ? w0.x : 0u; qa[kk][2] = ok0 ? w0.y : 0u;
                qa[kk][1] = ok1 ? w1.x : 0u; qa[kk][3] = ok1 ? w1.y : 0u;
            } else {
                qa[kk][0] = ok0 ? __ldcg(reinterpret_cast<const uint32_t*>(q0 + kk * 16 + c2)) : 0u;
                qa[kk][1] = ok1 ? __ldcg(reinterpret_cast<const uint32_t*>(q1 + kk * 16 + c2)) : 0u;
                qa[kk][2] = ok0 ? __ldcg(reinterpret_cast<const uint32_t*>(q0 + kk * 16 + 8 + c2)) : 0u;
                qa[kk][3] = ok1 ? __ldcg(reinterpret_cast<const uint32_t*>(q1 + kk * 16 + 8 + c2)) : 0u;
            }
        }
    }
    float o[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) { o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f; }
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;

    // The pages of a tile, one for each 16 rows (a page holds a multiple of 16); rows that nothing in the tile sees have none.
    auto tile_at = [&](int j, bool& summ) { summ = j < s_tiles; return summ ? s_t0 + j : t_t0 + j - s_tiles; };
    auto find_pages = [&](int j, int (&pg)[4]) {
        bool summ;
        const int x0 = tile_at(j, summ) * kPgTile;
        const int lo = summ ? see.s_lo : see.t_lo, hi = summ ? see.s_hi : see.t_hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = x0 + 16 * i;
            pg[i] = j < my1 && x < hi && x + 16 > lo ? paged_page(a, t.b, summ, x) : -3;
            if (pg[i] == -1 || pg[i] == -2) { atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_PAGE); pg[i] = -3; }
        }
    };
    // rows nobody sees and rows without a page come as zeros: they are masked, and their V must be finite
    auto load_tile = [&](int j, int stage, const int (&pg)[4]) {
        bool summ;
        const int x0 = tile_at(j, summ) * kPgTile;
        const int lo = summ ? see.s_lo : see.t_lo, hi = summ ? see.s_hi : see.t_hi;
        const uint32_t sk = sbase + stage * Cfg::kStageB, sv = sk + Cfg::kTileB;
        constexpr int kRowsPass = kPgThreads / Cfg::kVec, kPasses = kPgTile / kRowsPass;
        const int c16 = threadIdx.x % Cfg::kVec, rr = threadIdx.x / Cfg::kVec;
        const int in_page = (1 << a.page_shift) - 1;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int r = rr + i * kRowsPass, x = x0 + r;
            int page;
            if constexpr (kRowsPass <= 16) page = pg[i * kRowsPass / 16];
            else page = rr >= 16 ? pg[(i * kRowsPass / 16 + 1) & 3] : pg[i * kRowsPass / 16];
            const bool valid = page >= 0 && x >= lo && x < hi;
            const int64_t off = valid ? page * a.page_st + hk * a.head_st + (x & in_page) * a.row_st + c16 * 16 : 0;
            const uint32_t d = (uint32_t)(r * Cfg::kRowB + ((c16 ^ (Cfg::kVec == 4 ? (r >> 1) & 3 : r & 7)) << 4));
            pg_cp16(sk + d, a.kp + off, valid);
            pg_cp16(sv + d, a.vp + off, valid);
        }
        if constexpr (E4M3) {
            if (threadIdx.x < 8) {
                const int i = threadIdx.x & 3, x = x0 + 16 * i;
                const int page = i == 0 ? pg[0] : i == 1 ? pg[1] : i == 2 ? pg[2] : pg[3];
                const int64_t off = page >= 0 ? (((int64_t)page * a.Hkv + hk) << a.page_shift) + (x & in_page) : 0;
                pg_cp16(sk + 2 * Cfg::kTileB + threadIdx.x * 16, (threadIdx.x < 4 ? a.ke : a.ve) + off, page >= 0);
            }
        }
    };
    int pg[4];
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        if (my0 + s < my1) {
            find_pages(my0 + s, pg);
            load_tile(my0 + s, s, pg);
        }
        pg_commit();
    }
    find_pages(my0 + kStages - 1, pg);
    const int mi = lane >> 3, r8 = lane & 7;
    for (int j = my0; j < my1; ++j) {
        if (j + kStages - 1 < my1) load_tile(j + kStages - 1, (j - my0 + kStages - 1) % kStages, pg);
        pg_commit();
        find_pages(j + kStages, pg);                           // ahead of their use
        pg_wait<kStages - 1>();
        __syncthreads();
        const uint32_t sk = sbase + ((j - my0) % kStages) * Cfg::kStageB, sv = sk + Cfg::kTileB;
        const int wkey0 = warp * 16;
        // S (16 rows x 16 keys of this warp) = Q K^T
        float s[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) { s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f; }
        float fv[2][2];
        if constexpr (E4M3) {
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {              // 32 columns of 16 keys
                uint32_t kb[4];
                const int key = wkey0 + (mi >> 1) * 8 + r8, chunk = kk * 2 + (mi & 1);
                pg_ldsm(kb, sk + key * Cfg::kRowB + ((chunk ^ (Cfg::kVec == 4 ? (key >> 1) & 3 : key & 7)) << 4));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    pg_mma(s[i >> 1], qa[kk * 2 + (i & 1)], pg_two(kb[i]), pg_two(kb[i] >> 16));
            }
            const uint32_t se = sv + Cfg::kTileB + wkey0 + c2;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const uint32_t at = se + nt * 8, sh = (at & 2) * 8;
                const uint32_t ek = pg_ld_u32(at & ~3u) >> sh, ev = pg_ld_u32((at + kPgTile) & ~3u) >> sh;
                const float f0 = e8m0_scale(ek & 255), f1 = e8m0_scale(ek >> 8 & 255);
                s[nt][0] *= f0; s[nt][1] *= f1; s[nt][2] *= f0; s[nt][3] *= f1;
                fv[nt][0] = e8m0_scale(ev & 255); fv[nt][1] = e8m0_scale(ev >> 8 & 255);
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                uint32_t kb[4];
                const int key = wkey0 + (mi >> 1) * 8 + r8, chunk = kk * 2 + (mi & 1);
                pg_ldsm(kb, sk + key * Cfg::kRowB + ((chunk ^ (key & 7)) << 4));
                pg_mma(s[0], qa[kk], kb[0], kb[1]);
                pg_mma(s[1], qa[kk], kb[2], kb[3]);
            }
        }
        // each row's own range, online softmax in log2 units
        bool summ;
        const int x0 = tile_at(j, summ) * kPgTile + wkey0 + c2;
        const int lo0 = summ ? v0.s_lo : v0.t_lo, hi0 = summ ? v0.s_hi : v0.t_hi, lo1 = summ ? v1.s_lo : v1.t_lo, hi1 = summ ? v1.s_hi : v1.t_hi;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int x = x0 + nt * 8 + (e & 1);
                s[nt][e] = x >= (e < 2 ? lo0 : lo1) && x < (e < 2 ? hi0 : hi1) ? s[nt][e] * a.scale_log2 : -INFINITY;
            }
        float mx0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
        float mx1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1)); mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1)); mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
        const float mn0 = fmaxf(m0, mx0), mn1 = fmaxf(m1, mx1);
        const float al0 = (mn0 == -INFINITY) ? 1.f : ptx::ex2_approx(m0 - mn0), al1 = (mn1 == -INFINITY) ? 1.f : ptx::ex2_approx(m1 - mn1);
        const float sub0 = (mn0 == -INFINITY) ? 0.f : mn0, sub1 = (mn1 == -INFINITY) ? 0.f : mn1;
        m0 = mn0; m1 = mn1;
        float pr[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            pr[nt][0] = ptx::ex2_approx(s[nt][0] - sub0); pr[nt][1] = ptx::ex2_approx(s[nt][1] - sub0);
            pr[nt][2] = ptx::ex2_approx(s[nt][2] - sub1); pr[nt][3] = ptx::ex2_approx(s[nt][3] - sub1);
        }
        l0 = l0 * al0 + (pr[0][0] + pr[0][1]) + (pr[1][0] + pr[1][1]);
        l1 = l1 * al1 + (pr[0][2] + pr[0][3]) + (pr[1][2] + pr[1][3]);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) { o[i][0] *= al0; o[i][1] *= al0; o[i][2] *= al1; o[i][3] *= al1; }
        if constexpr (E4M3) {                                  // (the scale bytes of rows that nobody sees may be anything)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) pr[nt][e] = pr[nt][e] == 0.f ? 0.f : pr[nt][e] * fv[nt][e & 1];
        }
        uint32_t pa[4];
        pa[0] = ptx::pack_bf16x2(pr[0][0], pr[0][1]); pa[1] = ptx::pack_bf16x2(pr[0][2], pr[0][3]);
        pa[2] = ptx::pack_bf16x2(pr[1][0], pr[1][1]); pa[3] = ptx::pack_bf16x2(pr[1][2], pr[1][3]);
        // O += P V
        if constexpr (E4M3) {
            // o[2 i], o[2 i + 1]: the even and the odd columns of columns 16 i .. 16 i + 15
#pragma unroll
            for (int n2 = 0; n2 < D / 32; ++n2) {
                uint32_t vb[4];
                const int key = wkey0 + (mi & 1) * 8 + r8, chunk = n2 * 2 + (mi >> 1);
                pg_ldsm_t(vb, sv + key * Cfg::kRowB + ((chunk ^ (Cfg::kVec == 4 ? (key >> 1) & 3 : key & 7)) << 4));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w0 = __byte_perm(vb[2 * i], 0, 0x3120), w1 = __byte_perm(vb[2 * i + 1], 0, 0x3120);
                    pg_mma(o[4 * n2 + 2 * i], pa, pg_two(w0), pg_two(w1));
                    pg_mma(o[4 * n2 + 2 * i + 1], pa, pg_two(w0 >> 16), pg_two(w1 >> 16));
                }
            }
        } else {
#pragma unroll
            for (int n2 = 0; n2 < D / 16; ++n2) {
                uint32_t vb[4];
                const int key = wkey0 + (mi & 1) * 8 + r8, chunk = n2 * 2 + (mi >> 1);
                pg_ldsm_t(vb, sv + key * Cfg::kRowB + ((chunk ^ (key & 7)) << 4));
                pg_mma(o[2 * n2], pa, vb[0], vb[1]);
                pg_mma(o[2 * n2 + 1], pa, vb[2], vb[3]);
            }
        }
        __syncthreads();      // the stage is refilled by the load issued in the next iteration
    }
    pg_wait<0>();
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1); l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1); l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    // the four warps' results: 16 rows of (m, l) and 16 x D of O each
    __syncthreads();
    float* sm_o = reinterpret_cast<float*>(pgsm);                      // [4][16][D]
    float* sm_ml = sm_o + 4 * 16 * D;                                  // [4][16][2]
    float* ct_o = sm_ml + 4 * 16 * 2;                                  // this CTA's: [16][D]
    float* ct_ml = ct_o + 16 * D;                                      // [16][2]
    {
        float* r0 = sm_o + (warp * 16 + g0) * D;
        float* r1 = r0 + 8 * D;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if constexpr (E4M3) {
                const int d = i * 16 + c2 * 2;
                *reinterpret_cast<float4*>(r0 + d) = make_float4(o[2 * i][0], o[2 * i + 1][0], o[2 * i][1], o[2 * i + 1][1]);
                *reinterpret_cast<float4*>(r1 + d) = make_float4(o[2 * i][2], o[2 * i + 1][2], o[2 * i][3], o[2 * i + 1][3]);
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int d = i * 16 + u * 8 + c2;
                    *reinterpret_cast<float2*>(r0 + d) = make_float2(o[2 * i + u][0], o[2 * i + u][1]);
                    *reinterpret_cast<float2*>(r1 + d) = make_float2(o[2 * i + u][2], o[2 * i + u][3]);
                }
            }
        }
    }
    if ((lane & 3) == 0) {
        sm_ml[(warp * 16 + g0) * 2] = m0; sm_ml[(warp * 16 + g0) * 2 + 1] = l0;
        sm_ml[(warp * 16 + g0 + 8) * 2] = m1; sm_ml[(warp * 16 + g0 + 8) * 2 + 1] = l1;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < nrow * (D / 4); idx += kPgThreads) {
        const int g = idx / (D / 4), d = (idx - g * (D / 4)) * 4;
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, sm_ml[(w * 16 + g) * 2]);
        float L = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = sm_ml[(w * 16 + g) * 2];
            const float f = (mw == -INFINITY) ? 0.f : ptx::ex2_approx(mw - M);
            const float4 v = *reinterpret_cast<const float4*>(sm_o + (w * 16 + g) * D + d);
            L += sm_ml[(w * 16 + g) * 2 + 1] * f;
            acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
        }
        *reinterpret_cast<float4*>(ct_o + g * D + d) = acc;
        if (d == 0) { ct_ml[g * 2] = M; ct_ml[g * 2 + 1] = L; }
    }
    if (a.nsplit > 1) { ptx::cluster_arrive(); ptx::cluster_wait(); } else __syncthreads();
    // the cluster's CTAs share the output's elements
    const uint32_t so = ptx::smem_u32(ct_o), sml = ptx::smem_u32(ct_ml);
    for (int idx = split * kPgThreads + threadIdx.x; idx < nrow * (D / 4); idx += kPgThreads * a.nsplit) {
        const int g = idx / (D / 4), d = (idx - g * (D / 4)) * 4;
        float2 ml[kPgMaxSplit];
        float4 v[kPgMaxSplit];
#pragma unroll
        for (int w = 0; w < kPgMaxSplit; ++w)
            if (w < a.nsplit) {
                ml[w] = pg_ld_cluster2(ptx::mapa_shared(sml + g * 8, w));
                v[w] = pg_ld_cluster4(ptx::mapa_shared(so + (g * D + d) * 4, w));
            }
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < kPgMaxSplit; ++w) if (w < a.nsplit) M = fmaxf(M, ml[w].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kPgMaxSplit; ++w)
            if (w < a.nsplit) {
                const float f = (ml[w].x == -INFINITY) ? 0.f : ptx::ex2_approx(ml[w].x - M);
                L += ml[w].y * f;
                acc.x += v[w].x * f; acc.y += v[w].y * f; acc.z += v[w].z * f; acc.w += v[w].w * f;
            }
        const float inv = 1.f / L;
        const int64_t row = paged_row(a, t, t.x0 + g / heads);
        const int h = head0 + g % heads;
        if (!ksa_in_bounds(row >= 0 && row < a.rows && h < a.Hq, a.status)) continue;
        *reinterpret_cast<uint2*>(a.out + row * a.o_st + h * a.o_sh + d) =
            make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv), ptx::pack_bf16x2(acc.z * inv, acc.w * inv));
        if (d == 0) a.lse[(int64_t)h * a.rows + row] = (M + log2f(L)) * 0.6931471805599453f;
    }
    if (a.nsplit > 1) { ptx::cluster_arrive(); ptx::cluster_wait(); }      // no CTA leaves while another reads its results
}

template <int D, bool E4M3>
static cudaError_t setup_one()
{
    return cudaFuncSetAttribute(ksa_paged_attn_kernel<D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, PgCfg<D, E4M3>::kSmemBytes);
}
cudaError_t setup_paged_attn()
{
    for (cudaError_t e : {setup_one<128, false>(), setup_one<128, true>(), setup_one<64, false>(), setup_one<64, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

// CTAs of one cluster for a call of `units` query tiles at most: two CTAs of each SM, as far as there are key tiles to split
static int paged_splits(int64_t units, int64_t key_tiles, int num_sms)
{
    int n = 1;
    while (n < kPgMaxSplit && units * n * 2 <= 2 * num_sms && key_tiles >= 2 * n) n *= 2;
    return n;
}

cudaError_t launch_paged_attn(const PagedArgs& args, bool e4m3, int num_sms, cudaStream_t stream)
{
    PagedArgs a = args;
    a.tokens_per_tile = a.G <= 16 ? 16 / a.G : 1;
    a.head_blocks = (a.G + 15) / 16;
    // no tile without a row, none but a sequence's last of its kind with fewer than tokens_per_tile tokens
    const int64_t most = (int64_t)a.rows / a.tokens_per_tile + (int64_t)a.B * (a.m > 0 ? 2 : 1);
    const int64_t units = (most < a.rows ? most : a.rows) * a.Hkv * a.head_blocks;
    const int64_t rows = ((int64_t)a.text_cols + (a.m > 0 ? a.summ_cols : 0)) << a.page_shift;      // of a sequence, at most
    a.nsplit = paged_splits(units, rows / kPgTile, num_sms);
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.nsplit; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(units * a.nsplit)); cfg.blockDim = dim3(kPgThreads); cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = 2;
    auto go = [&](auto kernel, int smem) {
        cfg.dynamicSmemBytes = (size_t)smem;
        return cudaLaunchKernelEx(&cfg, kernel, a);
    };
    if (a.D == 128) return e4m3 ? go(ksa_paged_attn_kernel<128, true>, PgCfg<128, true>::kSmemBytes) : go(ksa_paged_attn_kernel<128, false>, PgCfg<128, false>::kSmemBytes);
    return e4m3 ? go(ksa_paged_attn_kernel<64, true>, PgCfg<64, true>::kSmemBytes) : go(ksa_paged_attn_kernel<64, false>, PgCfg<64, false>::kSmemBytes);
}

}  // namespace ksa
