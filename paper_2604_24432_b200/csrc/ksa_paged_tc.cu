// Attention of a run of new rows over the paged KV cache on the sm_100a tensor cores: pieces of prompts, drafted tokens.
//
// A CTA works on up to 256 query rows of one sequence and KV head, (token, query head of the group) each, as two tiles of 128
// (128 / group tokens), so that a key tile serves the whole group.  What they see is one range of summaries and one of text
// (Eq. 3; a summary: its own chunk), walked in tiles of 128 keys; where a call has too few query tiles for the device, the
// key tiles are split over a cluster's CTAs, whose results meet in distributed shared memory.
//
// Warp roles:
//   warps 0-3   query tile 0: load Q, softmax (one row per thread), O rescale, epilogue
//   warps 4-7   query tile 1
//   warp  8     TMA of the key tiles, one box a page, the pages looked up a tile ahead by a lane each
//   warp  9     issues S = Q K^T (tcgen05.mma, smem x smem)
//   warp 10     issues O += P V (P from TMEM)
//   warp 11     TMA of the value tiles (bf16 pages)
//   warps 12-15 (e4m3 pages) turn the tiles that warp 8 brings in 8 bits into f16 ones (or bf16, see below), a row's scale on the way
// TMEM: one score slot S [0,128) that the two query tiles take in turns, the 16-bit probabilities P0 [128,192), P1 [192,256),
// O0 [256,256+D), O1 [384,384+D).  The pipeline over the key tiles is that of the text-row kernel (ksa_text_tc.cu).
//
// e4m3 pages: the products are of f16 (one conversion for two values, one multiplication for their scale; as bf16 it takes three
// times the instructions, and the converting warps set the pace).  A row's scale is taken relative to the largest among the rows in
// view, which is found first: values are at most 448 * 2^7, and what underflows is below 2^-39 of the largest.  An e4m3 value has
// four significant bits, so rows whose scale is up to 2^28 smaller than the largest keep theirs.  Q becomes f16 by a power of two for
// each row; P as f16 is rounded eight times finer than as bf16, down to 2^-25 of the row's largest (see PtScale).  Where the scales in
// a CTA's view are further apart than that leaves room for (see PtTops), the same products are of bf16, which has the range: 200 rows
// over 36,864, 32/8 heads of 128: 65.7 and 79.6 us.
//
// Rows of a page that nothing in the tile sees may hold anything.  Scores of such keys are replaced by -inf; their V rows
// are overwritten with zeros in shared memory (0 * NaN would reach the accumulators): by warp 10 in the tiles that hold an end
// of a range, or by the converting warps.
//
// Every mbarrier wait is bounded, as in the other kernels: on timeout all roles leave their loops, copies in flight are waited
// for, the cluster's barriers are still passed, TMEM is freed.  (No test makes a wait of this kernel run out: the helper has one.)
//
// Measured: 1,152 rows over 36,864, 32/8 heads of 128, bf16: 72 us = 1,170 TFLOP/s of what is visible (83 us in a long loop, at the
// power cap; 128 of the query tiles are full ones, on 148 SMs); 1,000 and 1,024 rows over 16,001 and 7,168, causal, 16/16 heads:
// 183 us = 1,090 (214 us).  Tensor pipe 67 and 64 % of its cycles.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "ksa_launch.h"
#include "ksa_paged.h"
#include "ksa_ptx.cuh"
#include "ksa_wait.cuh"

namespace ksa {

using namespace ptx;

constexpr int kPtTile = 128;
// log2 units: by how much a score may outgrow the reference maximum before that moves, and what P stands above 2^(score - reference).
// bf16: P moves up to 2^12 past the first maximum (see ksa_text_tc.cu), and stands low, where bf16 keeps its bits: O is a sum of P V, which
// has to be within fp32 for V up to 2^128 and thousands of keys, and for V down to 2^-90.  f16 ends with 65,504 and loses bits below 2^-14, so P stays below 2^15 there, and as
// close to it as can be: it keeps 11 bits down to 2^-25 of the largest, and is 0 below 2^-36 of it.  (From 1 downwards, keys 18
// natural-log units below a single one in the same CTA's share came out as nothing.  900 rows over 36,864, 4/4 heads of 64:
// 32.7 and 32.9 us; 200 rows, 32/8 of 128: 65.2 and 66.3.)
template <bool E4M3> struct PtScale { static constexpr float kRescale = E4M3 ? 4.0f : 12.0f, kLift = E4M3 ? 11.0f : -30.0f, kUnit = E4M3 ? 0x1p-11f : 0x1p30f; };

template <int D, bool E4M3>
struct PtCfg {
    static constexpr int kThreads = E4M3 ? 512 : 384;
    // registers per thread after the hand-over: softmax, TMA / MMA, converting warps
    static constexpr int kRegsSoftmax = E4M3 ? 208 : 216, kRegsOther = E4M3 ? 40 : 72, kRegsConvert = 56;
    static_assert(8 * kRegsSoftmax + 4 * kRegsOther + (E4M3 ? 4 * kRegsConvert : 0) <= kThreads / 32 * ((65536 / kThreads) / 8 * 8), "register hand-over exceeds the CTA's allocation");
    static constexpr int kTileBytes = kPtTile * D * 2;
    static constexpr int kHalves = D / 64;           // 64-column (128-byte) swizzle panels
    static constexpr int kRawBytes = kPtTile * D;    // a tile in 8 bits
    static constexpr int kStagesK = E4M3 ? (D == 128 ? 2 : 3) : (D == 128 ? 3 : 5);
    static constexpr int kStagesV = E4M3 ? (D == 128 ? 2 : 3) : (D == 128 ? 2 : 5);
    static constexpr int kStagesRaw = E4M3 ? (D == 128 ? 2 : 6) : 0;
    static constexpr int kQOff = 0;
    static constexpr int kKOff = 2 * kTileBytes;
    static constexpr int kVOff = kKOff + kStagesK * kTileBytes;
    static constexpr int kRawOff = kVOff + kStagesV * kTileBytes;
    static constexpr int kBarOff = kRawOff + kStagesRaw * kRawBytes;
    // barrier slots
    static constexpr int kQFull = 0, kSFull = 2, kLoaded = 4, kPFull = 6, kPvDone = 8, kDrain = 10;
    static constexpr int kKFull = 12, kKEmpty = kKFull + kStagesK, kVFull = kKEmpty + kStagesK, kVEmpty = kVFull + kStagesV;
    static constexpr int kRawFull = kVEmpty + kStagesV, kRawEmpty = kRawFull + kStagesRaw;
    static constexpr int kNumBars = kRawEmpty + kStagesRaw;
    static constexpr int kSmemBytes = kBarOff + 8 * kNumBars + 64 + 1024;   // + slack for 1024-byte alignment
    // partial results, over Q, K and V once these are done with: O fp32 [256][D], (maximum, sum) [256], then where each row's output
    // and LSE go (offsets in elements; the first -1 for a row past the last)
    static constexpr int kPartMl = 256 * D * 4;
    static_assert(kPartMl + 256 * (8 + 16) <= kBarOff, "partial results fit over the tiles");
};

struct PagedMaps { CUtensorMap k, v; };

__device__ __forceinline__ void pt_named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void pt_st_shared4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 pt_ld_shared4(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 pt_ld_cluster4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 pt_ld_cluster2(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// e4m3: the largest scale bytes of K and of V among the rows in view, and whether the products are of bf16.  f16 has room for keys whose
// scale is up to 2^28 smaller than the largest (which other rows of the query tile may be the only ones to see).  A value row's share
// of the output is its probability times its scale, and P keeps bits down to 2^-25, so there it is 2^10, rows of zeros counted
// as the smallest (an attention sink of zeros leaves the output to probabilities of any size).
struct PtTops { uint32_t k, v; bool wide; };
__device__ __forceinline__ PtTops pt_tops(uint32_t at)
{
    uint32_t top[2] = {0u, 0u}, low[2] = {255u, 255u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {                              // by converting warp: K, V; largest, smallest
        const uint32_t w = ld_shared_u32(at + 4 * i);
        top[i & 1] = max(top[i & 1], w & 255u); low[i & 1] = min(low[i & 1], w >> 8);
    }
    return PtTops{top[0], top[1], (int)top[0] - (int)low[0] > 28 || (int)top[1] - (int)low[1] > 10};
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(PtCfg<D, E4M3>::kThreads, 1)
ksa_paged_tc_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedMaps maps)
{
    using Cfg = PtCfg<D, E4M3>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sQ = smem_base + Cfg::kQOff, sK = smem_base + Cfg::kKOff, sV = smem_base + Cfg::kVOff, sRaw = smem_base + Cfg::kRawOff;
    const uint32_t bars = smem_base + Cfg::kBarOff;
    const uint32_t tmem_slot = bars + 8 * Cfg::kNumBars;
    const uint32_t abort_addr = tmem_slot + 4;                 // (two words)
    const uint32_t tops = tmem_slot + 16;                       // e4m3: the largest and smallest scale bytes of K and of V, by converting warp
    auto bar = [&](int i) -> uint32_t { return bars + 8u * (uint32_t)i; };

    const int tid = threadIdx.x;
    const int warp = (int)__reduce_or_sync(0xffffffffu, (unsigned)tid >> 5);     // (uniform to the compiler)
    const int lane = tid & 31;

    if (tid == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(bar(Cfg::kQFull + t), 128);       // one arrival per thread that writes it
            mbar_init(bar(Cfg::kSFull + t), 1);
            mbar_init(bar(Cfg::kLoaded + t), 4);        // one arrival per softmax warp
            mbar_init(bar(Cfg::kPFull + t), 4);
            mbar_init(bar(Cfg::kPvDone + t), 1);
            mbar_init(bar(Cfg::kDrain + t), 1);
        }
        const int writers = E4M3 ? 4 : 1;               // converting warps, or the TMA's thread
        for (int st = 0; st < Cfg::kStagesK; ++st) { mbar_init(bar(Cfg::kKFull + st), writers); mbar_init(bar(Cfg::kKEmpty + st), 1); }
        for (int st = 0; st < Cfg::kStagesV; ++st) { mbar_init(bar(Cfg::kVFull + st), writers); mbar_init(bar(Cfg::kVEmpty + st), 1); }
        for (int st = 0; st < Cfg::kStagesRaw; ++st) { mbar_init(bar(Cfg::kRawFull + st), 1); mbar_init(bar(Cfg::kRawEmpty + st), 4); }
        st_shared_u32(abort_addr, 0u);
        st_shared_u32(abort_addr + 4, 0u);     // never raised: lets the teardown waits run while aborting
        fence_mbar_init();
    }
    if (warp == 8) {                           // one warp allocates all 512 TMEM columns (1 CTA per SM)
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ld_shared_u32(tmem_slot);
    if (a.beside != 2) pdl_wait();                          // (beside the kernel in front, which has waited for those before it)
    pdl_launch_dependents();

    const int unit = a.by_split((int)blockIdx.x), split = (int)blockIdx.x - unit * a.nsplit;
    const int item = a.by_heads(unit), hk = unit - item * a.Hkv;
    __shared__ __align__(16) PagedFound found;
    const PagedTile t = paged_tile<true, true, Cfg::kThreads>(a, item, found);   // up to 2 * per tokens
    const int per = a.tokens_per_tile / 2;
    if (t.b >= 0) {                                         // (the same for the whole cluster)
    PagedWalk<kPtTile> w;
    w.init(a, t, split, a.nsplit);
    const int T = w.j1 - w.j0;
    const int nh = T == 0 ? 0 : t.n > per ? 2 : 1;          // query tiles

    if (warp >= 12) {
        if constexpr (E4M3) {
            // ============================ 8-bit tiles to 16 bits ==========================
            setmaxnreg_dec<Cfg::kRegsConvert>();
            const int row = tid & 127;
            bool alive = true;
            int k_stage = 0, v_stage = 0, raw = 0;
            uint32_t k_phase = 0, v_phase = 0, raw_phase = 0;
            // the largest and the smallest scales of K and of V among the rows in view (rows of NaN and, of K, of zeros aside: the latter's
            // scores are 0 in any form): 16 rows at a time
            uint32_t top_k = 0, top_v = 0, low_k = ~0u, low_v = ~0u;
            for (int i = row; i < T * (kPtTile / 16); i += 128) {
                const auto tile = w.at(w.j0 + i / (kPtTile / 16));
                const int x = tile.x0 + i % (kPtTile / 16) * 16;
                if (!tile.sees_any(x, 16)) continue;
                const int page = paged_page(a, t.b, tile.summ, x);
                if (page < 0) continue;
                const int64_t at = (((int64_t)page * a.Hkv + hk) << a.page_shift) + (x & ((1 << a.page_shift) - 1));
                const uint4 k = __ldcg(reinterpret_cast<const uint4*>(a.ke + at)), v = __ldcg(reinterpret_cast<const uint4*>(a.ve + at));
                const uint32_t kw[4] = {k.x, k.y, k.z, k.w}, vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t in = 0u;                          // rows in view
#pragma unroll
                    for (int e = 0; e < 4; ++e) in |= tile.sees(x + 4 * c + e) ? 0xffu << (8 * e) : 0u;
                    const uint32_t ik = in & ~__vcmpeq4(kw[c], 0xffffffffu), iv = in & ~__vcmpeq4(vw[c], 0xffffffffu);
                    top_k = __vmaxu4(top_k, kw[c] & ik); top_v = __vmaxu4(top_v, vw[c] & iv);
                    low_k = __vminu4(low_k, kw[c] | ~ik | __vcmpleu4(kw[c], 0x11111111u)); low_v = __vminu4(low_v, vw[c] | ~iv);
                }
            }
            auto publish = [&](uint32_t top, uint32_t low, uint32_t to) {
                top = __vmaxu2(top >> 8 & 0x00ff00ffu, top & 0x00ff00ffu); low = __vminu2(low >> 8 & 0x00ff00ffu, low & 0x00ff00ffu);
                top = __reduce_max_sync(0xffffffffu, max(top >> 16, top & 0xffffu));
                low = __reduce_min_sync(0xffffffffu, min(low >> 16, low & 0xffffu));
                if (lane == 0) st_shared_u32(to, top | low << 8);
            };
            publish(top_k, low_k, tops + 8 * (warp - 12));
            publish(top_v, low_v, tops + 8 * (warp - 12) + 4);
            pt_named_barrier(2, 448);                          // with the softmax and the MMA warps, who need them too
            const PtTops top = pt_tops(tops);
            // 2^(e - top + 7), as f16 twice or (for bf16) as fp32; 255: NaN
            auto factor = [&](uint32_t e, uint32_t largest) {
                const int p = (int)e - (int)largest + 7;
                if (top.wide) return e == 255u ? 0x7fc00000u : p >= -126 ? (uint32_t)(p + 127) << 23 : 0u;
                const uint32_t h = e == 255u ? 0x7e00u : p >= -14 ? (uint32_t)(p + 15) << 10 : p >= -24 ? 1u << (p + 24) : 0u;
                return h | h << 16;
            };
            // this thread's row of tile j: its factors (found a tile ahead), 0xffffffff where nobody sees it
            auto scales = [&](int j, uint32_t& fk, uint32_t& fv) {
                fk = fv = 0xffffffffu;
                if (j >= w.j1) return;
                const auto tile = w.at(j);
                const int x = tile.x0 + row;
                if (!tile.sees(x)) return;
                const int page = paged_page(a, t.b, tile.summ, x);
                if (page < 0) return;
                const int64_t at = (((int64_t)page * a.Hkv + hk) << a.page_shift) + (x & ((1 << a.page_shift) - 1));
                fk = factor(__ldcg(a.ke + at), top.k);
                fv = factor(__ldcg(a.ve + at), top.v);
            };
            auto convert = [&](uint32_t full, uint32_t empty, uint32_t empty_parity, uint32_t dst, uint32_t f) {
                if (alive) alive = __all_sync(0xffffffffu, bounded_wait(bar(Cfg::kRawFull + raw), raw_phase, abort_addr, a.status, kStatusWaitKvFull));
                if (alive) alive = __all_sync(0xffffffffu, bounded_wait(empty, empty_parity, abort_addr, a.status, kStatusWaitKvEmpty));
                if (!alive) return;
                // A warp takes its 32 rows four (D = 64: eight) at a time, 16 bytes a lane.  Lanes 0-3 of eight have a row's one half and
                // lanes 4-7 the next row's other half: neither the reads nor the writes, whose 16-byte places are permuted by the
                // row's last bits, meet in a bank.
                const uint32_t src = sRaw + raw * Cfg::kRawBytes + (row & 96) * D;
                constexpr int kStep = 512 / D;                      // rows of a step
                const int r0 = D == 128 ? (lane >> 4) * 2 + (lane >> 2 & 1) : lane >> 2;
                const int half = D == 128 ? (lane >> 3 & 1) ^ (lane >> 2 & 1) : 0, c = lane & 3;
                const uint32_t at = src + r0 * D + half * 64 + c * 16, to = dst + half * 16384 + ((row & 96) + r0) * 128;
                const bool all = __all_sync(0xffffffffu, f != 0xffffffffu);
                auto rows = [&](auto wide) {
#pragma unroll
                for (int i = 0; i < 32 / kStep; ++i) {
                    const uint4 y = pt_ld_shared4(at + i * kStep * D);
                    const uint32_t g = __shfl_sync(0xffffffffu, f, r0 + i * kStep);
                    const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
                    uint32_t z[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (wide) {
                            const float2 p = e4m3x2_to_f32(yw[e] & 0xffffu), q = e4m3x2_to_f32(yw[e] >> 16);
                            const float f32 = __uint_as_float(g);
                            z[2 * e] = pack_bf16x2(p.x * f32, p.y * f32); z[2 * e + 1] = pack_bf16x2(q.x * f32, q.y * f32);
                        } else {
                            e4m3x4_to_f16(yw[e], z[2 * e], z[2 * e + 1]);
                            z[2 * e] = mul_f16x2(z[2 * e], g); z[2 * e + 1] = mul_f16x2(z[2 * e + 1], g);
                        }
                    }
                    if (!all && g == 0xffffffffu) {                 // nobody sees the row: it may hold anything
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = 0u;
                    }
                    const int x = (r0 + i * kStep) & 7;
                    pt_st_shared4(to + i * kStep * 128 + (((c * 2) ^ x) << 4), z[0], z[1], z[2], z[3]);
                    pt_st_shared4(to + i * kStep * 128 + (((c * 2 + 1) ^ x) << 4), z[4], z[5], z[6], z[7]);
                }
                };
                if (top.wide) rows(std::true_type{}); else rows(std::false_type{});
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) { mbar_arrive(full); mbar_arrive(bar(Cfg::kRawEmpty + raw)); }
                if (++raw == Cfg::kStagesRaw) { raw = 0; raw_phase ^= 1u; }
            };
            // K a tile ahead of V: a K stage is free as soon as its scores are loaded, a V stage only after the product behind the
            // softmax, and the next scores must not wait for that
            uint32_t fk, fv, fv_before = 0;
            scales(w.j0, fk, fv);
            for (int j = w.j0; j <= w.j1 && T > 0 && alive; ++j) {
                uint32_t nk, nv;
                scales(j + 1, nk, nv);
                if (j < w.j1) {
                    convert(bar(Cfg::kKFull + k_stage), bar(Cfg::kKEmpty + k_stage), k_phase ^ 1u, sK + k_stage * Cfg::kTileBytes, fk);
                    if (++k_stage == Cfg::kStagesK) { k_stage = 0; k_phase ^= 1u; }
                }
                if (j > w.j0) {
                    convert(bar(Cfg::kVFull + v_stage), bar(Cfg::kVEmpty + v_stage), v_phase ^ 1u, sV + v_stage * Cfg::kTileBytes, fv_before);
                    if (++v_stage == Cfg::kStagesV) { v_stage = 0; v_phase ^= 1u; }
                }
                fv_before = fv; fk = nk; fv = nv;
            }
            if (a.nsplit > 1) { __syncwarp(); cluster_arrive(); cluster_wait(); cluster_arrive(); cluster_wait(); }
        }
    } else if (warp >= 8) {
        setmaxnreg_dec<Cfg::kRegsOther>();
        if (warp == 8 || (warp == 11 && !E4M3)) {
            // =============================== TMA producers ===============================
            // bf16: warp 8 brings the K tiles, warp 11 the V tiles; e4m3: warp 8 brings K and V tiles in turn.  A page is
            // one box (a panel of 64 columns of it in bf16), each by a lane of its own.
            const bool is_v = warp == 11;
            const int stages = E4M3 ? Cfg::kStagesRaw : is_v ? Cfg::kStagesV : Cfg::kStagesK;
            const uint32_t ring = E4M3 ? sRaw : is_v ? sV : sK;
            const uint32_t full0 = bar(E4M3 ? Cfg::kRawFull : is_v ? Cfg::kVFull : Cfg::kKFull), empty0 = bar(E4M3 ? Cfg::kRawEmpty : is_v ? Cfg::kVEmpty : Cfg::kKEmpty);
            constexpr int kBytes = E4M3 ? Cfg::kRawBytes : Cfg::kTileBytes;
            const int pages = kPtTile >> a.page_shift;       // of a tile
            if (lane == 0) { prefetch_tensormap(&maps.k); prefetch_tensormap(&maps.v); }
            // page of lane's rows of tile j; num_pages (a box of zeros) where nobody sees any of them
            auto find = [&](int j) {
                if (j >= w.j1 || lane >= pages) return a.num_pages;
                const auto tile = w.at(j);
                const int x = tile.x0 + (lane << a.page_shift);
                if (!tile.sees_any(x, 1 << a.page_shift)) return a.num_pages;
                const int page = paged_page(a, t.b, tile.summ, x);
                if (page < 0) { atomicCAS(a.status, 0, KSA_PAGED_STATUS_BAD_PAGE); return a.num_pages; }
                return page;
            };
            int stage = 0;
            uint32_t phase = 0, armed_mask = 0, armed_parity = 0;
            bool alive = true;
            int page = find(w.j0), page_before = 0;
            // (e4m3: K a tile ahead of V, as the converting warps take them)
            for (int j = w.j0; j < w.j1 + (E4M3 && T > 0 ? 1 : 0) && alive; ++j) {
                const int next = find(j + 1);
                for (int u = 0; u < (E4M3 ? 2 : 1) && alive; ++u) {
                    if (E4M3 && (u == 0 ? j == w.j1 : j == w.j0)) continue;
                    const uint32_t full = full0 + 8u * stage;
                    alive = __all_sync(0xffffffffu, bounded_wait(empty0 + 8u * stage, phase ^ 1u, abort_addr, a.status, kStatusWaitKvEmpty));
                    if (!alive) break;
                    if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)kBytes);
                    armed_mask |= 1u << stage;
                    armed_parity = (armed_parity & ~(1u << stage)) | (phase << stage);
                    __syncwarp();
                    if (lane < pages) {
                        const CUtensorMap* map = is_v || u == 1 ? &maps.v : &maps.k;
                        const uint32_t rows0 = (uint32_t)lane << a.page_shift;
                        if constexpr (E4M3) {
                            tma_load_4d(ring + stage * kBytes + rows0 * D, map, full, 0, 0, hk, u == 1 ? page_before : page);
                        } else {
#pragma unroll
                            for (int h = 0; h < Cfg::kHalves; ++h) tma_load_4d(ring + stage * kBytes + h * 16384 + rows0 * 128, map, full, h * 64, 0, hk, page);
                        }
                    }
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                }
                page_before = page;
                page = next;
            }
            // leave no copy in flight behind, whoever gives up on it later on
            for (int st = 0; st < stages; ++st)
                if (armed_mask & (1u << st)) bounded_wait(full0 + 8u * st, (armed_parity >> st) & 1u, abort_addr + 4, a.status, kStatusWaitKvFull);
        } else if (warp != 11) {
            // =============================== MMA issuers =================================
            constexpr uint32_t hi = smem_desc_hi_sw128(1024);
            const uint32_t leader = elect_one();
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            bool bf16 = !E4M3;
            if constexpr (E4M3) { pt_named_barrier(2, 448); bf16 = __all_sync(0xffffffffu, pt_tops(tops).wide); }
            bool alive = true;
            auto wait = [&](uint32_t b, uint32_t parity, int code) {
                if (alive) alive = __all_sync(0xffffffffu, bounded_wait(b, parity, abort_addr, a.status, code));
            };
            uint32_t stage = 0, ring_phase = 0, phase0 = 0, phase1 = 0;
            if (warp == 9) {
                const uint32_t idesc = bf16 ? make_idesc_bf16(128, 128, false) : make_idesc_f16(128, 128, false);
                const uint32_t q_lo = smem_desc_lo(sQ, 16), k_lo = smem_desc_lo(sK, 16);
                int before = -1;                            // query tile whose scores stand in the slot
                for (int j = 0; j < T && alive; ++j) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (u == 1 && nh == 1) break;
                        if (j == 0) wait(bar(Cfg::kQFull + u), 0, kStatusWaitQFull);
                        if (u == 0) wait(bar(Cfg::kKFull) + 8u * stage, ring_phase, kStatusWaitKvFull);
                        // the slot: the scores before are in their group's registers
                        if (before == 0) { wait(bar(Cfg::kLoaded), phase0, kStatusWaitPFull); phase0 ^= 1u; }
                        else if (before == 1) { wait(bar(Cfg::kLoaded + 1), phase1, kStatusWaitPFull); phase1 ^= 1u; }
                        if (!alive) break;
                        before = u;
                        tc_fence_after();
                        const uint32_t qd = q_lo + (uint32_t)(u * (Cfg::kTileBytes >> 4)), kd = k_lo + stage * (uint32_t)(Cfg::kTileBytes >> 4);
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t off = (uint32_t)((kk >> 2) * 16384 + (kk & 3) * 32) >> 4;
                            mma_ss_warp(leader, tm, qd + off, kd + off, hi, idesc, kk > 0 ? 1u : 0u);
                        }
                        tc_commit_warp(leader, bar(Cfg::kSFull + u));
                    }
                    if (++stage == (uint32_t)Cfg::kStagesK) { stage = 0; ring_phase ^= 1u; }
                }
            } else {
                const uint32_t idesc = bf16 ? make_idesc_bf16(128, D, true) : make_idesc_f16(128, D, true);
                const uint32_t v_lo = smem_desc_lo(sV, 16384);   // MN-major: 64-column panels 16 KB apart, groups of 8 keys 1 KB
                for (int j = 0; j < T && alive; ++j) {
                    wait(bar(Cfg::kVFull) + 8u * stage, ring_phase, kStatusWaitKvFull);
                    if constexpr (!E4M3) {
                        const auto tile = w.at(w.j0 + j);
                        if (alive && !tile.sees_all()) {       // rows that nobody sees: zeros
                            const uint32_t base = sV + stage * Cfg::kTileBytes + (uint32_t)(lane & 7) * 16u;
                            for (int r = lane >> 3; r < kPtTile; r += 4)
                                if (!tile.sees(tile.x0 + r))
#pragma unroll
                                    for (int h = 0; h < Cfg::kHalves; ++h) pt_st_shared4(base + h * 16384 + r * 128, 0u, 0u, 0u, 0u);
                            fence_proxy_async();
                            __syncwarp();
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (u == 1 && nh == 1) break;
                        wait(bar(Cfg::kPFull + u), u ? phase1 : phase0, kStatusWaitPFull);
                        if (u) phase1 ^= 1u; else phase0 ^= 1u;
                        if (!alive) break;
                        tc_fence_after();
                        const uint32_t vd = v_lo + stage * (uint32_t)(Cfg::kTileBytes >> 4);
#pragma unroll
                        for (int kk = 0; kk < kPtTile / 16; ++kk)
                            mma_ts_warp(leader, tm + 256u + u * 128u, tm + 128u + u * 64u + kk * 8u, vd + (uint32_t)((kk * 2048) >> 4), hi, idesc, (j > 0 || kk > 0) ? 1u : 0u);
                        tc_commit_warp(leader, bar(Cfg::kPvDone + u));
                    }
                    if (++stage == (uint32_t)Cfg::kStagesV) { stage = 0; ring_phase ^= 1u; }
                }
            }
            // drain the tensor pipe before TMEM is released
            const uint32_t drain = bar(Cfg::kDrain + (warp == 9 ? 0 : 1));
            tc_commit_warp(leader, drain);
            bounded_wait(drain, 0, abort_addr + 4, a.status, kStatusWaitOFull);
        }
        if (a.nsplit > 1) { __syncwarp(); cluster_arrive(); cluster_wait(); cluster_arrive(); cluster_wait(); }
    } else {
        setmaxnreg_inc<Cfg::kRegsSoftmax>();
        // =============================== softmax warpgroups =========================
        const int u = warp >> 2;
        const int row = tid & 127;
        const uint32_t lane_sel = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_sel;                                   // the score slot
        const uint32_t tP = tmem + lane_sel + 128u + (uint32_t)(u * 64);
        const uint32_t tO = tmem + lane_sel + 256u + (uint32_t)(u * 128);
        const int tokens = min(per, t.n - u * per);                            // of this query tile (0 or less: none)
        float m_used = -INFINITY, l_run = 0.f;
        const int nrow = max(tokens, 0) * a.G;
        const int r_in = min(row, max(nrow - 1, 0));                           // rows past the last mimic it; never stored
        const int in_tile = a.by_group(r_in), token = u * per + in_tile;
        bool is_summ;
        const int x = paged_token(a, t, token, is_summ);
        const int64_t prow = t.mixed ? t.row0 + token : paged_row(a, t, x);
        const int head = hk * a.G + r_in - in_tile * a.G;
        const bool valid = row < nrow;
        bool alive = true;
        float q_back = 1.f, v_back = 1.f;                                      // e4m3: what the scores and O are to be multiplied with
        // ---- Q: a warp's 32 rows, K-major with 128-byte swizzle; D / 8 lanes bring a row (a row per thread took 4.4 us of a
        // CTA's 11.7 with one key tile) ----
        constexpr int kLanesQ = D / 8, kRowsPassQ = 32 / kLanesQ;
        const int qc = lane % kLanesQ, qr0 = lane / kLanesQ;
        uint4 y[kLanesQ];
        if (u < nh) {
            const int64_t off = prow * a.q_st + head * a.q_sh;
#pragma unroll
            for (int i = 0; i < kLanesQ; ++i)
                y[i] = __ldcg(reinterpret_cast<const uint4*>(a.q + __shfl_sync(0xffffffffu, off, i * kRowsPassQ + qr0) + qc * 8));
        }
        bool wide = false;                                   // e4m3: the products are of bf16
        if constexpr (E4M3) {
            pt_named_barrier(2, 448);                        // the largest scales are known
            const PtTops top = pt_tops(tops);
            wide = __all_sync(0xffffffffu, top.wide);
            q_back = e8m0_factor(top.k) * 0.0078125f;        // (K and V stand 2^7 times larger)
            v_back = e8m0_factor(top.v) * 0.0078125f;
        }
        if (u < nh) {
            if constexpr (E4M3) {                            // the row's largest value taken to 2^8 or more (below 2^9)
                const float back = q_back;
#pragma unroll
                for (int i = 0; i < kLanesQ; ++i) {
                    uint32_t top = __vmaxu2(__vmaxu2(y[i].x & 0x7fff7fffu, y[i].y & 0x7fff7fffu), __vmaxu2(y[i].z & 0x7fff7fffu, y[i].w & 0x7fff7fffu));
#pragma unroll
                    for (int o = kLanesQ / 2; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const int e = min(max((int)(max(top >> 16, top & 0xffffu) >> 7) - 8, 1), 253);
                    const float f = __uint_as_float((uint32_t)(254 - e) << 23);
                    auto two = [&](uint32_t& z) {
                        const float lo = __uint_as_float(z << 16) * f, hi = __uint_as_float(z & 0xffff0000u) * f;
                        z = wide ? pack_bf16x2(lo, hi) : pack_f16x2(lo, hi);
                    };
                    two(y[i].x); two(y[i].y); two(y[i].z); two(y[i].w);
                    const int mine = __shfl_sync(0xffffffffu, e, lane % kRowsPassQ * kLanesQ);
                    if (lane / kRowsPassQ == i) q_back = __uint_as_float((uint32_t)mine << 23) * back;      // (of this thread's own row)
                }
            }
            const uint32_t d = sQ + u * Cfg::kTileBytes + (qc >> 3) * 16384 + (row & 96) * 128;
#pragma unroll
            for (int i = 0; i < kLanesQ; ++i) {
                const int r = i * kRowsPassQ + qr0;
                pt_st_shared4(d + r * 128 + (((qc ^ r) & 7) << 4), y[i].x, y[i].y, y[i].z, y[i].w);
            }
            fence_proxy_async();
            mbar_arrive(bar(Cfg::kQFull + u));
        }
        if (u < nh) {
            const PagedView see = paged_view(a, is_summ, x);
            // (a normal number: a query of zeros over small keys would make it 0, and what is masked is -inf before it is scaled; scores
            // that it multiplies stay next to 0, or far apart, all the same)
            const float scale_log2 = E4M3 ? fminf(fmaxf(a.scale_log2 * q_back, 0x1p-126f), 0x1.fffffep127f) : a.scale_log2;
            uint32_t sf_phase = 0, pv_phase = 0;
            int rel_k = 0, rel_v = 0;                        // the stages handed back next, by the last query tile's first thread
            const bool releaser = (tid & 127) == 0 && u == nh - 1;
            auto release_k = [&]() { mbar_arrive_relaxed(bar(Cfg::kKEmpty + rel_k)); if (++rel_k == Cfg::kStagesK) rel_k = 0; };
            auto release_v = [&]() { mbar_arrive_relaxed(bar(Cfg::kVEmpty + rel_v)); if (++rel_v == Cfg::kStagesV) rel_v = 0; };
            bool s_ok = false;                               // the scores of this tile are known to be there
            for (int j = 0; j < T; ++j) {
                bool ok;
                if (!__all_sync(0xffffffffu, s_ok)) {
                    ok = bounded_wait(bar(Cfg::kSFull + u), sf_phase, abort_addr, a.status, kStatusWaitSFull);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) { alive = false; break; }
                }
                sf_phase ^= 1u;
                tc_fence_after();
                uint32_t s[128];
                {
                    uint32_t (&c0)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[0]);
                    uint32_t (&c1)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[32]);
                    uint32_t (&c2)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[64]);
                    uint32_t (&c3)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[96]);
                    tmem_ld32(tS + 0, c0); tmem_ld32(tS + 32, c1); tmem_ld32(tS + 64, c2); tmem_ld32(tS + 96, c3);
                }
                if (releaser) release_k();                   // both query tiles' products with K(j) are done
                tc_wait_ld();
                // the scores are in registers: the slot may take the next ones
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_relaxed(bar(Cfg::kLoaded + u));
                // the row's own range, where the tile holds an end of some row's
                const auto tile = w.at(w.j0 + j);
                const int ca = (tile.summ ? see.s_lo : see.t_lo) - tile.x0, cb = (tile.summ ? see.s_hi : see.t_hi) - tile.x0;    // visible columns
                if (__any_sync(0xffffffffu, ca > 0 || cb < kPtTile)) {
                    const uint32_t width = (uint32_t)max(cb - ca, 0);
#pragma unroll
                    for (int c = 0; c < 128; ++c)
                        if ((uint32_t)(c - ca) >= width) s[c] = 0xff800000u;   // -inf
                }
                // row maximum, two new scores per instruction
                float mx0 = fmax3(__uint_as_float(s[0]), __uint_as_float(s[1]), __uint_as_float(s[2]));
                float mx1 = fmax3(__uint_as_float(s[3]), __uint_as_float(s[4]), __uint_as_float(s[5]));
                float mx2 = fmax3(__uint_as_float(s[6]), __uint_as_float(s[7]), __uint_as_float(s[8]));
                float mx3 = fmax3(__uint_as_float(s[9]), __uint_as_float(s[10]), __uint_as_float(s[11]));
#pragma unroll
                for (int c = 12; c < 124; c += 8) {
                    mx0 = fmax3(mx0, __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                    mx1 = fmax3(mx1, __uint_as_float(s[c + 2]), __uint_as_float(s[c + 3]));
                    mx2 = fmax3(mx2, __uint_as_float(s[c + 4]), __uint_as_float(s[c + 5]));
                    mx3 = fmax3(mx3, __uint_as_float(s[c + 6]), __uint_as_float(s[c + 7]));
                }
                mx0 = fmax3(mx0, __uint_as_float(s[124]), __uint_as_float(s[125]));
                mx1 = fmax3(mx1, __uint_as_float(s[126]), __uint_as_float(s[127]));
                const float mx_sc = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * scale_log2;
                // lazy rescale: the reference max only moves when some row of the warp outgrew it
                const bool need_any = __any_sync(0xffffffffu, mx_sc > m_used + PtScale<E4M3>::kRescale);
                float alpha = 1.f;
                if (need_any) {
                    const float m_new = fmaxf(m_used, mx_sc);
                    alpha = (m_new == -INFINITY) ? 1.f : ex2_approx(m_used - m_new);
                    m_used = m_new;
                    l_run *= alpha;
                }
                const float neg_m = (m_used == -INFINITY) ? 0.f : PtScale<E4M3>::kLift - m_used;
                const float2 sc2 = make_float2(scale_log2, scale_log2);
                const float2 nm2 = make_float2(neg_m, neg_m);
                bool pv_ok = false;                           // the product before is known to be done
                float2 la = make_float2(0.f, 0.f), lb = make_float2(0.f, 0.f);
                auto exponentials = [&](auto half) {           // (half: whether as f16)
#pragma unroll
                for (int q = 0; q < 64; ++q) {
                    const float2 z = ffma2(make_float2(__uint_as_float(s[2 * q]), __uint_as_float(s[2 * q + 1])), sc2, nm2);
                    float2 pr;
                    pr.x = ex2_approx(z.x); pr.y = ex2_approx(z.y);
                    if (q & 1) lb = fadd2(lb, pr); else la = fadd2(la, pr);
                    if (q == 48 && j > 0) pv_ok = mbar_test_wait(bar(Cfg::kPvDone + u), pv_phase);
                    s[q] = half ? pack_f16x2(pr.x, pr.y) : pack_bf16x2(pr.x, pr.y);
                }
                };
                if constexpr (E4M3) {
                    if (wide) exponentials(std::false_type{}); else exponentials(std::true_type{});
                } else {
                    exponentials(std::false_type{});
                }
                l_run += (la.x + la.y) + (lb.x + lb.y);
                if (j > 0) {
                    // O_u += P_u V(j-1) has read P_u and written O_u
                    if (!__all_sync(0xffffffffu, pv_ok)) {
                        ok = bounded_wait(bar(Cfg::kPvDone + u), pv_phase, abort_addr, a.status, kStatusWaitPvDone);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) { alive = false; break; }
                    }
                    pv_phase ^= 1u;
                    if (releaser) release_v();               // V(j-1)
                    tc_fence_after();
                }
                s_ok = j + 1 < T && mbar_test_wait(bar(Cfg::kSFull + u), sf_phase);
                {
                    uint32_t (&p0)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[0]);
                    uint32_t (&p1)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[32]);
                    tmem_st32(tP + 0, p0); tmem_st32(tP + 32, p1);
                }
                if (need_any && j > 0) {
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(tO + c * 32, o);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tmem_st32(tO + c * 32, o);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_relaxed(bar(Cfg::kPFull + u));
            }
            if (alive) {
                const bool ok = bounded_wait(bar(Cfg::kPvDone + u), pv_phase, abort_addr, a.status, kStatusWaitOFull);
                alive = __all_sync(0xffffffffu, ok);
                tc_fence_after();
            }
        }
        if (a.nsplit == 1) {
            // ---- epilogue: O / l -> bf16 at the row's place, LSE ----
            if (u < nh && alive) {
                const float inv_l = v_back / l_run;
                const bool store = valid && ksa_in_bounds(prow >= 0 && prow < a.rows && head < a.Hq, a.status);
                // a row stands in one lane: four lanes exchange 64 bytes of their rows, so that a store touches 8 lines, not 32
                const int64_t off = store ? prow * a.o_st + (int64_t)head * a.o_sh : -1;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tO + c * 32, o);
                    tc_wait_ld();
                    uint4 pk[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        pk[e].x = pack_bf16x2(__uint_as_float(o[8 * e]) * inv_l, __uint_as_float(o[8 * e + 1]) * inv_l);
                        pk[e].y = pack_bf16x2(__uint_as_float(o[8 * e + 2]) * inv_l, __uint_as_float(o[8 * e + 3]) * inv_l);
                        pk[e].z = pack_bf16x2(__uint_as_float(o[8 * e + 4]) * inv_l, __uint_as_float(o[8 * e + 5]) * inv_l);
                        pk[e].w = pack_bf16x2(__uint_as_float(o[8 * e + 6]) * inv_l, __uint_as_float(o[8 * e + 7]) * inv_l);
                    }
                    quad_transpose(pk, lane);                             // pk[e]: 16 bytes of the group's row e
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t at = __shfl_sync(0xffffffffu, off, (lane & 28) + e);
                        if (at >= 0) *reinterpret_cast<uint4*>(a.out + at + c * 32 + (lane & 3) * 8) = pk[e];
                    }
                }
                if (store) a.lse[(int64_t)head * a.rows + prow] = (m_used + log2f(l_run * PtScale<E4M3>::kUnit)) * 0.6931471805599453f;
                tc_fence_before();
            }
        } else {
            // ---- partial results into shared memory, summed up over the cluster, a share of the rows by each CTA ----
            pt_named_barrier(1, 256);                         // both query tiles' products have read their K, V and Q
            const uint32_t part_o = smem_base, part_ml = smem_base + Cfg::kPartMl, part_to = part_ml + 256 * 8;
            // e4m3: O / sum / 8, and the sum in the maximum's place, as log2: times V's scale O itself may be beyond fp32 (whose
            // largest is 1.4 times that of the format's values), and so may a sum of several CTAs' O / sum
            float part_m = m_used, part_l = l_run, part_f = 1.f;
            if constexpr (E4M3) {
                part_f = (l_run == 0.f) ? 0.f : v_back * (0.125f / l_run);
                part_m = (l_run == 0.f) ? -INFINITY : m_used + log2f(l_run * PtScale<E4M3>::kUnit);
                part_l = (l_run == 0.f) ? 0.f : 1.f;
            }
            if (tokens > 0) {
                const uint32_t d = part_o + (uint32_t)((u * 128 + row) * D * 4);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    if (u < nh) {
                        tmem_ld32(tO + c * 32, o);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) if (E4M3) o[e] = __float_as_uint(__uint_as_float(o[e]) * part_f);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0u;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e)               // (neighbouring rows on different banks)
                        pt_st_shared4(d + (uint32_t)((c * 8 + (e ^ (row & 7))) * 16), o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                }
                asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(part_ml + (u * 128 + row) * 8), "f"(part_m), "f"(part_l) : "memory");
                const bool store = valid && ksa_in_bounds(prow >= 0 && prow < a.rows && head < a.Hq, a.status);
                const uint64_t off = store ? (uint64_t)(prow * a.o_st + (int64_t)head * a.o_sh) : ~0ull, lse = (uint64_t)((int64_t)head * a.rows + prow);
                pt_st_shared4(part_to + (u * 128 + row) * 16, (uint32_t)off, (uint32_t)(off >> 32), (uint32_t)lse, (uint32_t)(lse >> 32));
                tc_fence_before();
            }
            __syncwarp();
            cluster_arrive(); cluster_wait();
            // D / 4 lanes a row, kMerge rows and two CTAs at a time so that the reads of the other CTAs' memory overlap
            constexpr int kLanes = D / 4, kRowsPass = 256 / kLanes, kMerge = 4;
            const int rows0 = per * a.G, total = t.n * a.G, c4 = tid % kLanes, step = kRowsPass * a.nsplit;
            for (int i0 = split * kRowsPass + tid / kLanes; i0 < total; i0 += kMerge * step) {
                uint32_t at[kMerge], pr[kMerge];
                float M[kMerge], L[kMerge];
                float4 acc[kMerge];
#pragma unroll
                for (int r = 0; r < kMerge; ++r) {
                    const int i = min(i0 + r * step, total - 1);
                    pr[r] = i < rows0 ? i : 128 + i - rows0;                          // row of the partial results
                    at[r] = part_o + (uint32_t)(pr[r] * (D * 4) + ((c4 & ~7) + ((c4 ^ pr[r]) & 7)) * 16);
                    M[r] = -INFINITY; L[r] = 0.f;
                    acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                for (int s0 = 0; s0 < a.nsplit; s0 += 2) {
                    float2 ml[2][kMerge];
                    float4 v[2][kMerge];
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const uint32_t other = mapa_shared(smem_base, min(s0 + s, a.nsplit - 1)) - smem_base;
#pragma unroll
                        for (int r = 0; r < kMerge; ++r) { ml[s][r] = pt_ld_cluster2(part_ml + pr[r] * 8 + other); v[s][r] = pt_ld_cluster4(at[r] + other); }
                    }
                    if (s0 + 1 == a.nsplit) {                                         // (the last of an odd number comes alone)
#pragma unroll
                        for (int r = 0; r < kMerge; ++r) ml[1][r].x = -INFINITY;
                    }
#pragma unroll
                    for (int r = 0; r < kMerge; ++r) {
                        const float m = fmax3(M[r], ml[0][r].x, ml[1][r].x), base = (m == -INFINITY) ? 0.f : m;
                        const float al = ex2_approx(M[r] - base), f0 = ex2_approx(ml[0][r].x - base), f1 = ex2_approx(ml[1][r].x - base);
                        M[r] = m;
                        L[r] = fmaf(L[r], al, fmaf(ml[0][r].y, f0, ml[1][r].y * f1));
                        acc[r].x = fmaf(acc[r].x, al, fmaf(v[0][r].x, f0, v[1][r].x * f1)); acc[r].y = fmaf(acc[r].y, al, fmaf(v[0][r].y, f0, v[1][r].y * f1));
                        acc[r].z = fmaf(acc[r].z, al, fmaf(v[0][r].z, f0, v[1][r].z * f1)); acc[r].w = fmaf(acc[r].w, al, fmaf(v[0][r].w, f0, v[1][r].w * f1));
                    }
                }
#pragma unroll
                for (int r = 0; r < kMerge; ++r) {
                    if (i0 + r * step >= total) break;
                    const uint4 to = pt_ld_shared4(part_to + pr[r] * 16);             // where the row's output and LSE go
                    const int64_t off = (int64_t)((uint64_t)to.y << 32 | to.x), lse = (int64_t)((uint64_t)to.w << 32 | to.z);
                    if (off < 0) continue;
                    const float inv = (E4M3 ? 8.f : 1.f) / L[r];
                    *reinterpret_cast<uint2*>(a.out + off + c4 * 4) = make_uint2(pack_bf16x2(acc[r].x * inv, acc[r].y * inv), pack_bf16x2(acc[r].z * inv, acc[r].w * inv));
                    if (c4 == 0) a.lse[lse] = (M[r] + log2f(E4M3 ? L[r] : L[r] * PtScale<E4M3>::kUnit)) * 0.6931471805599453f;
                }
            }
            __syncwarp();
            cluster_arrive(); cluster_wait();                 // no CTA leaves while another reads its results
        }
    }
    }

    if (a.beside == 2) pdl_wait();                          // whoever waits for this kernel finds both done
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
}

template <int D, bool E4M3>
static cudaError_t setup_one()
{
    return cudaFuncSetAttribute(ksa_paged_tc_kernel<D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, PtCfg<D, E4M3>::kSmemBytes);
}
cudaError_t setup_paged_tc()
{
    for (cudaError_t e : {setup_one<128, false>(), setup_one<128, true>(), setup_one<64, false>(), setup_one<64, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

// CTAs of one cluster for a call of `units` query tiles at most.  Joining the parts costs some 5 us of a CTA's time, so the key
// tiles are split where SMs would stand idle: 16 query tiles of 17 (65) key tiles each on 1, 2, 4, 8 CTAs: 34.5, 28.1, 22.9,
// 43 us (104, 63, 41, 63 us; clusters of eight CTAs that fill an SM find few places).  More than two take seven tenths of the
// SMs at most, since clusters of them leave SMs of a group of SMs over: 32 query tiles of some 60 key tiles on 2, 3, 4: 43.5,
// 37.6, 40.7 us; 16 on 3, 4, 6, 8: 34.3, 30.9, 28.1, 48.7 us.  And in two where a call of a few rounds
// holds several sequences, whose lengths differ, the longest first: two sequences of 17,000 and 8,192 rows, 16/16 heads: 206 and
// 186 us, eight of 1 to 577 new rows over up to 31,000: 71 and 57.5 us; but one sequence, 144 even query tiles: 74 and 96 us.
static int tc_splits(int64_t units, int64_t key_tiles, int seqs, int num_sms)
{
    for (int n : {6, 4, 3})
        if (units * n * 10 <= num_sms * 7 && key_tiles >= (n > 4 ? 32 : 16)) return n;
    if (units * 2 <= num_sms && key_tiles >= 12) return 2;
    return seqs > 1 && units * 2 <= 4 * num_sms && key_tiles >= 32 ? 2 : 1;
}

// Tiles of a call: query tokens of a CTA, and the key tiles that one may see at most
static int tc_tokens(const PagedArgs& a) { return 2 * (kPtTile / a.G); }
static int64_t tc_key_tiles(const PagedArgs& a)
{
    const int64_t text = std::min((int64_t)a.text_cols << a.page_shift, ((int64_t)a.C + 2) * a.kk + tc_tokens(a));
    return (text + (a.m > 0 ? (int64_t)a.summ_cols << a.page_shift : 0)) / kPtTile;
}

// Rounds of CTAs on the SMs: some 6 us each (and 10 for the call), and 2.4 us a key tile with e4m3 pages, 1.3 with bf16 ones
float paged_tc_us(const PagedArgs& args, bool e4m3, int num_sms)
{
    PagedArgs a = args;
    a.tokens_per_tile = tc_tokens(a);
    const int64_t key_tiles = tc_key_tiles(a), n = tc_splits(paged_most_tiles(a) * a.Hkv, key_tiles, a.B, num_sms);
    const int64_t tiles = std::max((a.rows + a.tokens_per_tile - 1) / a.tokens_per_tile, a.B) * (int64_t)a.Hkv;
    const float per_tile = (e4m3 ? 2.4f : 1.3f) * (a.D == 128 ? 1.0f : 0.7f);
    return 10.0f + (float)((tiles * n + num_sms - 1) / num_sms) * (6.0f + per_tile * std::max(1.0f, (float)key_tiles / (float)n));
}

cudaError_t launch_paged_tc(const PagedArgs& args, bool e4m3, int num_sms, PagedEncode encode, cudaStream_t stream)
{
    PagedArgs a = args;
    a.tokens_per_tile = tc_tokens(a);                         // of a CTA: two query tiles
    a.head_blocks = 1;
    a.by_tile = PagedDiv::by(a.tokens_per_tile); a.by_group = PagedDiv::by(a.G);
    const int64_t units = paged_most_tiles(a) * a.Hkv;
    a.nsplit = tc_splits(units, tc_key_tiles(a), a.B, num_sms);
    a.by_split = PagedDiv::by(a.nsplit);
    a.by_heads = PagedDiv::by(a.Hkv);
    PagedMaps maps;
    const int box_bytes = e4m3 ? a.D : 128;
    const CUtensorMapSwizzle swizzle = e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B;
    if (!encode_pages(encode, &maps.k, a.kp, a, e4m3, box_bytes, 1 << a.page_shift, swizzle) || !encode_pages(encode, &maps.v, a.vp, a, e4m3, box_bytes, 1 << a.page_shift, swizzle))
        return cudaErrorInvalidValue;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.nsplit; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(units * a.nsplit)); cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = 2;
    auto go = [&](auto kernel, int threads, int smem) {
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = (size_t)smem;
        return cudaLaunchKernelEx(&cfg, kernel, a, maps);
    };
    if (a.D == 128) {
        if (e4m3) return go(ksa_paged_tc_kernel<128, true>, PtCfg<128, true>::kThreads, PtCfg<128, true>::kSmemBytes);
        return go(ksa_paged_tc_kernel<128, false>, PtCfg<128, false>::kThreads, PtCfg<128, false>::kSmemBytes);
    }
    if (e4m3) return go(ksa_paged_tc_kernel<64, true>, PtCfg<64, true>::kThreads, PtCfg<64, true>::kSmemBytes);
    return go(ksa_paged_tc_kernel<64, false>, PtCfg<64, false>::kThreads, PtCfg<64, false>::kSmemBytes);
}

}  // namespace ksa
