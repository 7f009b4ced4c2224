// Attention of one new token per stream over the slots that a group of streams shares, computed once
// for the whole group (sirllm_attend_shared): the query heads of all streams of the group that share a
// K/V head are the rows of one product,
//     S = Q K^T [rows x slots],   P = 2^(scale log2e S - reference),   O = P V,
// and every row's (reference, sum of P, O) over a stretch of the slots goes to the workspace, where
// join_kernel adds it to what attend_kernel makes of the stream's own slots.
//
// Read once for up to 256 rows, K and V cost 4 * rows operations per element: HBM's bound up to about 250
// rows, the tensor core's beyond.  tcgen05 for both products: 128 rows on the lanes, S and O in tensor
// memory; P goes back there as the left operand of the second product, V is its right operand as it
// lies in memory ([slot][element], rows of the product along the columns of V).
// One persistent CTA per SM takes an equal stretch of the line of all units' tiles (128 slots).  Two lanes of
// work (S, P, O each) keep the tensor core and the exponentials busy at once: with more than 128 rows
// they are two blocks of rows over the same tiles, else the even and the odd tiles of one block, whose
// results are joined at the end of the stretch.  Warp 0 loads (TMA, a ring of K and V tiles), warp 1
// issues the products, four warps per lane own one row per thread.
// The reference moves only when a score passes it by more than 2^8 (bf16; fp16: the weights stand 2^11 to
// 2^15 above the reference, see attend_kernel), so O is rarely rescaled.  Sums, references and O are
// fp32; P is rounded to 16 bits on its way into the second product.
// Measured, 64 streams x 32 heads on 8 x 15873 slots: 24 us of the call's 50 (floor 10.4, the products).  A tile takes both
// lanes 3900 cycles: weights 2400, then products and the next scores 1470, in turns; the tensor core alone would
// take 2050, the exponentials alone (32768 at 16 a cycle) 2048.  The rest is the start (thousands of cycles to the
// first scores, mostly instructions on their way into the cache) and the end.
// Whole tiles only: what is left of the shared slots (fewer than 128) attend_kernel reads itself, so
// nothing here is masked and no slot behind the shared ones is read.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tcgen05.cuh"

namespace sirllm {

namespace {

constexpr int kThreads = 384;       // loads, products, two idle warps, 2 x 4 warps of rows
constexpr int kRowThreads = 256;
constexpr int kPanelBytes = 128 * 128;  // 64 elements of 128 rows or slots, 128-byte swizzle
constexpr int kSmemRoom = 224 * 1024;
template <int kPanels>
constexpr int kStagesOf = kPanels == 1 ? 10 : (kSmemRoom - 2 * kPanels * kPanelBytes) / (kPanels * kPanelBytes);
constexpr uint32_t kScoreCol = 0, kOutCol = 256, kLaneCols = 128;  // tensor memory: S (and P) and O of the two lanes

constexpr float kLowest = -3.4028235e38f;

template <bool kBf16>
constexpr float kSetBelow = kBf16 ? 0.f : 11.f;
template <bool kBf16>
constexpr float kMoveAt = kBf16 ? 8.f : 15.f;

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar,
                                            uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5}], "
        "[%2], %6;" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "l"(policy)
        : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::
            "r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// Right operand with the product's columns contiguous: panels of 64 columns kPanelBytes apart, groups of
// 8 slots 1024 bytes apart.
__device__ __forceinline__ uint32_t columns_lo(uint32_t addr) {
    return ((addr & 0x3FFFFu) >> 4) | ((uint32_t)(kPanelBytes >> 4) << 16);
}
// one lane of the warp, the same every time; the compiler knows that it is one
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// left operand from tensor memory
__device__ __forceinline__ void mma_f16_tmem(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b_lo), "r"(idesc), "r"((uint32_t)accumulate), "r"(kOperandHi)
        : "memory");
}
// 32 columns, without waiting
__device__ __forceinline__ void tmem_ask32(uint32_t (&r)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_give32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// eight values, one sector of memory
__device__ __forceinline__ void store8(float* at, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t out;
    if (kBf16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(out) : "f"(hi), "f"(lo));
    return out;
}

__device__ __forceinline__ int group_tiles(const PrefixParams& p, int g) {
    const int n = p.shared_len[g];
    return n < 0 || n > p.capacity ? 0 : prefix_slots(n) / kPrefixTile;
}

// A CTA's way along its stretch of the line, unit by unit.
struct Stretch {
    int left;         // tiles of the stretch from here on
    int g, u;         // group, unit of the group
    int t0, tiles;    // first tile here, tiles of a unit of this group
    __device__ __forceinline__ int count() const { return min(left, tiles - t0); }
    __device__ __forceinline__ void next(const PrefixParams& p) {
        left -= count();
        t0 = 0;
        if (left > 0 && ++u == p.n_kv_heads * p.plan.units) {
            u = 0;
            for (tiles = 0; tiles == 0;) {
                if (++g >= p.n_groups) {  // (the lengths changed under the call)
                    left = 0;
                    return;
                }
                tiles = group_tiles(p, g);
            }
        }
    }
};

// kPair: two blocks of rows over the same tiles; else one block, its even and its odd tiles.
// kPanels: panels of 64 elements of a head.
template <bool kBf16, bool kPair, int kPanels>
__global__ void __launch_bounds__(kThreads, 1)
prefix_kernel(const PrefixParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
              const __grid_constant__ CUtensorMap map_v) {
    constexpr int kStageBytes = kPanels * kPanelBytes;
    constexpr int kStages = kStagesOf<kPanels>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages];
    __shared__ __align__(8) uint64_t q_full[2], q_empty[2];     // the two buffers of queries
    __shared__ __align__(8) uint64_t s_full[2], p_full[2][2], o_full[2], o_empty, drained;
    __shared__ float2 stats[kPrefixRows];
    __shared__ Stretch first;
    __shared__ int tiles_per_cta;
    __shared__ uint32_t tmem_base;
    __shared__ volatile int gave_up;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t q_at = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_bytes = kPanels * kPanelBytes;              // a buffer of queries
    const uint32_t ring = q_at + 2 * q_bytes;

    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i][0], 4);
            mbar_init(&p_full[i][1], 4);
            mbar_init(&o_full[i], 1);
        }
        mbar_init(&o_empty, kRowThreads / 32);
        mbar_init(&drained, 1);
        mbar_init_fence();
        gave_up = 0;
    }
    if (warp == 1) tmem_alloc<1>(&tmem_base);
    if (tid == 0) {
        prefetch_map(&map_q);
        prefetch_map(&map_k);
        prefetch_map(&map_v);
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_base;

    grid_dependency_wait();
    if (warp == 2) {
        // the line: its length, and this CTA's stretch
        const int per_group = p.n_kv_heads * p.plan.units;
        const int T0 = lane < p.n_groups ? group_tiles(p, lane) : 0;
        int total = __reduce_add_sync(0xFFFFFFFFu, T0 * per_group);
        for (int g0 = 32; g0 < p.n_groups; g0 += 32)
            total += __reduce_add_sync(0xFFFFFFFFu, g0 + lane < p.n_groups ? group_tiles(p, g0 + lane) * per_group : 0);
        const int per = max((total + (int)gridDim.x - 1) / (int)gridDim.x, 2);
        const int begin = (int)min((int64_t)blockIdx.x * per, (int64_t)total);
        Stretch w;
        w.left = min(per, total - begin);
        int before = 0;
        for (int g0 = 0; g0 < p.n_groups && before <= begin; g0 += 32) {
            const int g = g0 + lane;
            const int T = g0 == 0 ? T0 : g < p.n_groups ? group_tiles(p, g) : 0;
            int upto = T * per_group;
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= o) upto += v;
            }
            const int start = before + upto - T * per_group;
            if (w.left > 0 && T > 0 && begin >= start && begin < before + upto) {  // one lane, once
                w.g = g;
                w.u = (begin - start) / T;
                w.t0 = begin - start - w.u * T;
                w.tiles = T;
                first = w;
            }
            before += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
        if (lane == 0) tiles_per_cta = per;
        if (w.left <= 0 && lane == 0) {
            w.left = 0;
            first = w;
        }
    }
    __syncthreads();
    grid_launch_dependents();

    // A wait that runs out raises the flag and every role leaves; the others see it or run out too.  Of whole
    // warps, which leave as one: lanes poll at different times, and what follows (a lane elected among 32, loads and
    // stores of tensor memory) wants them all.
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        bool there = false;
        for (uint32_t i = 0; i < kSpinLimit && !there; ++i) {
            there = mbar_try_wait(bar, parity);
            if (!there && gave_up) break;
        }
        if (!there) gave_up = 1;
        return __all_sync(0xFFFFFFFFu, there);
    };
    constexpr int kTilesAtOnce = kPair ? 1 : 2;  // tiles that the two lanes take together

    if (warp < 4) {
        if (warp == 0) {  // ---- loads
            const bool issuer = elect_one();
            // K and V that only one CTA reads shall not push other things out of L2 (this kernel's
            // instructions among them: fetching them from HBM costs microseconds at every start)
            uint64_t policy;
            if (p.plan.units == 1)
                asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
            else
                asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            uint32_t q_phase = 0;
            int buf = 0, q_asked = 0;
            auto feed = [&]() -> bool {
                for (Stretch w = first; w.left > 0; w.next(p)) {
                    const int kv_head = w.u / p.plan.units, block0 = kPair ? (w.u - kv_head * p.plan.units) * 2 : 0;
                    // queries: both blocks, or the one block into the buffers in turn
                    for (int b = 0; b < (kPair ? 2 : 1); ++b) {
                        const int q_buf = kPair ? b : buf;
                        if (!wait(&q_empty[q_buf], q_phase ^ 1u)) return false;
                        if (issuer) {
                            mbar_expect_tx(&q_full[q_buf], p.q_box_bytes * kPanels);
                            for (int i = 0; i < kPanels; ++i)
                                tma_load_4d(q_at + q_buf * q_bytes + i * kPanelBytes, &map_q, i * 64, 0, kv_head,
                                            w.g * p.stream_group + (block0 + b) * p.plan.block_streams,
                                            smem_u32(&q_full[q_buf]));
                        }
                        ++q_asked;
                    }
                    if (kPair || buf == 1) q_phase ^= 1u;
                    buf ^= 1;
                    const int plane = w.g * p.stream_group * p.planes_per_stream + p.layer_plane + kv_head;
                    for (int t = 0; t < w.count(); ++t)
                        for (int kv = 0; kv < 2; ++kv) {
                            if (!wait(&empty[stage], phase ^ 1u)) return false;
                            if (issuer) {
                                mbar_expect_tx(&full[stage], kStageBytes);
                                for (int i = 0; i < kPanels; ++i)
                                    tma_load_3d(ring + stage * kStageBytes + i * kPanelBytes, kv == 0 ? &map_k : &map_v,
                                                i * 64, (w.t0 + t) * kPrefixTile, plane, smem_u32(&full[stage]), policy);
                            }
                            if (issued < kStages) ++issued;
                            if (++stage == kStages) {
                                stage = 0;
                                phase ^= 1u;
                            }
                        }
                }
                return true;
            };
            if (!feed() && issuer) {  // gave up: let the loads in flight land
                for (int i = 0; i < issued; ++i)
                    for (uint32_t parity = 0; parity < 2; ++parity) mbar_wait_bounded(&full[i], parity, 1u << 14);
                for (int i = 0; i < 2 && i < q_asked; ++i)
                    for (uint32_t parity = 0; parity < 2; ++parity) mbar_wait_bounded(&q_full[i], parity, 1u << 14);
            }
        } else if (warp == 1) {  // ---- products
            auto multiply = [&]() {
                const uint32_t type = (1u << 4) | ((uint32_t)kBf16 << 7) | ((uint32_t)kBf16 << 10) | (8u << 24);  // 128 rows
                const uint32_t s_desc = type | (16u << 17);                                       // 128 slots
                const int out_cols = (p.head_dim + 15) / 16 * 16;
                const uint32_t o_desc = type | (1u << 16) | ((uint32_t)(out_cols >> 3) << 17);    // V: columns contiguous
                // job n is tile n / 2 of lane n % 2 (pair), or tile n of lane n % 2; its K and V are two stages
                int k_stage = 0, v_stage = 1;
                uint32_t k_phase = 0, v_phase = 0, p_phase[2] = {0, 0}, q_phase = 0, o_phase = 0;
                int buf = 0;
                bool begun = false;
                auto step = [&](int& stage, uint32_t& phase) {
                    stage += 2;
                    if (stage >= kStages) {
                        stage -= kStages;
                        phase ^= 1u;
                    }
                };
                for (Stretch w = first; w.left > 0; w.next(p)) {
                    const int tiles = w.count(), jobs = kPair ? 2 * tiles : tiles;
                    auto scores = [&](int n) -> bool {  // S of job n
                        const int ln = n & 1;
                        if (kPair ? n < 2 : n == 0) {
                            if (!wait(&q_full[kPair ? ln : buf], q_phase)) return false;
                        }
                        if (!kPair || ln == 0) {
                            if (!wait(&full[k_stage], k_phase)) return false;
                        }
                        tmem_fence_after();
                        const uint32_t a = operand_lo(q_at + (kPair ? ln : buf) * q_bytes);
                        const uint32_t b = operand_lo(ring + k_stage * kStageBytes);
                        const uint32_t d = tmem + kScoreCol + ln * kLaneCols;
                        if (elect_one()) {
#pragma unroll
                            for (int i = 0; i < kPanels * 4; ++i) {  // (what lies behind head_dim is zeros)
                                const uint32_t off = (uint32_t)(i >> 2) * (kPanelBytes >> 4) + (uint32_t)(i & 3) * 2;
                                mma_f16<1>(d, a + off, b + off, s_desc, i > 0);
                            }
                            if (!kPair || ln == 1) mma_commit<1>(&empty[k_stage]);
                            if (kPair ? n >= jobs - 2 : n == jobs - 1) mma_commit<1>(&q_empty[kPair ? ln : buf]);
                            mma_commit<1>(&s_full[ln]);
                        }
                        if (!kPair || ln == 1) step(k_stage, k_phase);
                        return true;
                    };
                    for (int n = 0; n < 2 && n < jobs; ++n)
                        if (!scores(n)) return;
                    if (begun && !wait(&o_empty, o_phase)) return;  // the last unit's results have been read
                    if (begun) o_phase ^= 1u;
                    begun = true;
                    for (int n = 0; n < jobs; ++n) {
                        const int ln = n & 1;
                        const uint32_t b = columns_lo(ring + v_stage * kStageBytes);
                        const uint32_t d = tmem + kOutCol + ln * kLaneCols, a = tmem + kScoreCol + ln * kLaneCols;
                        const bool more = n > 1;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (!wait(&p_full[ln][half], p_phase[ln])) return;
                            if (half == 0 && (!kPair || ln == 0)) {
                                if (!wait(&full[v_stage], v_phase)) return;
                            }
                            tmem_fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int i = half * 4; i < half * 4 + 4; ++i)
                                    mma_f16_tmem(d, a + i * 8, b + i * (2048 >> 4), o_desc, i > 0 || more);
                                if (half == 1) {
                                    if (!kPair || ln == 1) mma_commit<1>(&empty[v_stage]);
                                    if (n + 2 >= jobs) mma_commit<1>(&o_full[ln]);
                                }
                            }
                        }
                        p_phase[ln] ^= 1u;
                        if (!kPair || ln == 1) step(v_stage, v_phase);
                        if (n + 2 < jobs && !scores(n + 2)) return;
                    }
                    if (kPair || buf == 1) q_phase ^= 1u;
                    buf ^= 1;
                }
            };
            multiply();
            if (elect_one()) mma_commit<1>(&drained);
        }
    } else {  // ---- one row of a lane per thread
        const int quarter = warp & 3, ln = (warp - 4) >> 2, row = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)quarter << 21);
        const uint32_t s_at = lanes + kScoreCol + ln * kLaneCols, o_at = lanes + kOutCol + ln * kLaneCols;
        uint32_t s_phase = 0, o_phase[2] = {0, 0};
        const float scale = p.scale_log2;
        const uint32_t flip = scale < 0.f ? 0x80000000u : 0u;  // the largest score is the smallest product then
        bool ok = true;
        // (a warp that gave up goes on to meet the others at their barriers)
        for (Stretch w = first; w.left > 0; w.next(p)) {
            const int kv_head = w.u / p.plan.units, block0 = kPair ? (w.u - kv_head * p.plan.units) * 2 : 0;
            const int block = block0 + (kPair ? ln : 0);
            const int used = max(0, min(p.plan.block_streams, p.stream_group - block * p.plan.block_streams)) * p.heads;
            const bool any = quarter * 32 < used;   // rows of this warp that are somebody's
            const int tiles = w.count();
            float m = kNegHuge, l = 0.f;
            bool fresh = true;
            // Twice over a row's scores, 64 columns at a time, in loops: what is not in the instruction cache
            // comes in at 250 cycles and more per 8 instructions (unrolled over the row, the first tile of a call
            // took 2 us more; in steps of 32 columns the others 0.3 us more).
            for (int t = kPair ? 0 : ln; t < tiles && ok; t += kTilesAtOnce, fresh = false) {
                ok = wait(&s_full[ln], s_phase);
                if (!ok) break;
                s_phase ^= 1u;
                tmem_fence_after();
                if (any) {
                    float top[4] = {kLowest, kLowest, kLowest, kLowest};
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        uint32_t s[2][32];
                        tmem_ask32(s[0], s_at + i * 64);
                        tmem_ask32(s[1], s_at + i * 64 + 32);
                        tmem_wait_loads();
#pragma unroll
                        for (int j = 0; j < 64; j += 2)
                            top[(j >> 1) & 3] = fmaxf(fmaxf(top[(j >> 1) & 3], __uint_as_float(s[j >> 5][j & 31] ^ flip)),
                                                      __uint_as_float(s[j >> 5][(j & 31) + 1] ^ flip));
                    }
                    const float high = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * fabsf(scale);
                    if (__any_sync(0xFFFFFFFFu, high > m + kMoveAt<kBf16>)) {
                        const float up = fmaxf(m, high - kSetBelow<kBf16>);
                        const float f = ex2_approx(m - up);
                        m = up;
                        l *= f;
                        // the products so far are done: S came after them
#pragma unroll 1
                        for (int i = 0; !fresh && i * 32 < p.head_dim; ++i) {
                            uint32_t o[32];
                            tmem_ask32(o, o_at + i * 32);
                            tmem_wait_loads();
#pragma unroll
                            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                            tmem_give32(o_at + i * 32, o);
                        }
                    }
                    const uint64_t scale2 = pack2(scale, scale), minus2 = pack2(-m, -m);
                    uint64_t sum[2] = {0, 0};
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        uint32_t s[2][32], w16[32];
                        tmem_ask32(s[0], s_at + i * 64);
                        tmem_ask32(s[1], s_at + i * 64 + 32);
                        tmem_wait_loads();
#pragma unroll
                        for (int j = 0; j < 64; j += 2) {
                            float e0, e1;
                            unpack2(fma2(pack2(__uint_as_float(s[j >> 5][j & 31]), __uint_as_float(s[j >> 5][(j & 31) + 1])),
                                         scale2, minus2), e0, e1);
                            e0 = ex2_approx(e0);
                            e1 = ex2_approx(e1);
                            sum[(j >> 1) & 1] = add2(sum[(j >> 1) & 1], pack2(e0, e1));
                            w16[j >> 1] = pack16<kBf16>(e0, e1);
                        }
                        tmem_give32(s_at + i * 32, w16);  // half of the weights, over scores that have been read
                        tmem_wait_stores();
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&p_full[ln][i]);
                    }
                    float s0, s1;
                    unpack2(add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                } else {
                    tmem_fence_before();
                    __syncwarp();
                    if (lane < 2) mbar_arrive(&p_full[ln][lane]);
                }
            }
            // ---- the unit's part -----------------------------------------------------------------
            const int lanes_used = kPair || tiles > 1 ? 2 : 1;
            const int64_t place =
                ((int64_t)w.g * p.n_kv_heads * p.plan.units + w.u + blockIdx.x) * p.plan.rows + row + (kPair ? ln * kPrefixRows : 0);
            for (int x = 0; x < 2; ++x)
                if (x < lanes_used && (!kPair || x == ln) && ok) {
                    ok = wait(&o_full[x], o_phase[x]);
                    o_phase[x] ^= 1u;
                }
            if (w.t0 == 0 && tid == kThreads - 1) {  // where the unit's parts are
                const int behind = w.tiles - w.count();
                p.plan.parts[w.g * p.n_kv_heads * p.plan.units + w.u] =
                    make_int2(blockIdx.x, 1 + (behind + tiles_per_cta - 1) / tiles_per_cta);
            }
            tmem_fence_after();
            float* dst = p.plan.part_o + place * p.head_dim;
            if (kPair) {
                if (any && ok) {
#pragma unroll 1
                    for (int i = 0; i * 32 < p.head_dim; ++i) {
                        uint32_t o[32];
                        tmem_ask32(o, o_at + i * 32);
                        tmem_wait_loads();
                        if (row < used) {
#pragma unroll
                            for (int j = 0; j < 32; j += 8)
                                if (i * 32 + j < p.head_dim) store8(dst + i * 32 + j, o + j);
                        }
                    }
                    if (row < used) p.plan.part_ml[place] = make_float2(m, l);
                }
            } else {
                // the even and the odd tiles into one; each of a row's two threads takes half of the columns
                if (ln == 1) stats[row] = make_float2(m, l);
                asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
                float2 f;
                if (ln == 0) {
                    const float2 odd = stats[row];
                    const float up = fmaxf(m, odd.x);
                    f = make_float2(ex2_approx(m - up), ex2_approx(odd.x - up));
                    stats[row] = f;
                    if (row < used && ok) p.plan.part_ml[place] = make_float2(up, l * f.x + odd.y * f.y);
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
                if (ln == 1) f = stats[row];
                if (any && ok) {
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        const int col = ln * 64 + i * 32;
                        if (col >= p.head_dim) break;
                        uint32_t o[32], q[32];
                        tmem_ask32(o, lanes + kOutCol + col);
                        tmem_ask32(q, lanes + kOutCol + kLaneCols + col);
                        tmem_wait_loads();
                        if (row < used) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                float v = __uint_as_float(o[j]) * f.x;
                                if (lanes_used == 2) v = fmaf(__uint_as_float(q[j]), f.y, v);
                                o[j] = __float_as_uint(v);
                            }
#pragma unroll
                            for (int j = 0; j < 32; j += 8)
                                if (col + j < p.head_dim) store8(dst + col + j, o + j);
                        }
                    }
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&o_empty);
        }
    }
    tmem_fence_before();
    __syncthreads();
    // products still under way use shared memory and tensor memory
    if (warp == 1) {
        if (lane == 0) {
            bool done = false;
            for (uint32_t i = 0; i < kNapLimit && !done; ++i) done = mbar_nap(&drained, 0);
            if (!done) gave_up = 1;
        }
        __syncwarp();
    }
    __syncthreads();
    tmem_fence_after();
    if (warp == 1) tmem_free<1>(tmem);
    if (tid == 0 && gave_up) atomicOr(p.status, SIRLLM_STATUS_TIMEOUT);
}

template <bool kBf16, bool kPair, int kPanels>
cudaError_t launch_one(const PrefixParams& p, const DeviceProps& dp, const CUtensorMap& q, const CUtensorMap& k,
                   const CUtensorMap& v, cudaStream_t st) {
    static unsigned char allowed[kMaxDevices];
    auto kernel = prefix_kernel<kBf16, kPair, kPanels>;
    cudaError_t e = allow_max_dynamic_smem((const void*)kernel, dp, allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(dp.n_sm < kAttendMaxCtas ? dp.n_sm : kAttendMaxCtas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = 1024 + (size_t)(2 + kStagesOf<kPanels>) * kPanels * kPanelBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, q, k, v);
}

template <bool kBf16, bool kPair>
cudaError_t launch(const PrefixParams& p, const DeviceProps& dp, const CUtensorMap& q, const CUtensorMap& k,
                   const CUtensorMap& v, cudaStream_t st) {
    return p.head_dim <= 64 ? launch_one<kBf16, kPair, 1>(p, dp, q, k, v, st) : launch_one<kBf16, kPair, 2>(p, dp, q, k, v, st);
}

}  // namespace

bool prefix_plan(const sirllm_config& c, int32_t stream_group, int32_t n_heads, PrefixPlan* plan) {
    const int heads = n_heads / c.n_kv_heads;
    if (heads > kPrefixRows || c.head_dim > 128) return false;
    *plan = PrefixPlan{};
    plan->block_streams = stream_group < kPrefixRows / heads ? stream_group : kPrefixRows / heads;
    plan->blocks = (stream_group + plan->block_streams - 1) / plan->block_streams;
    plan->pair = plan->blocks > 1;
    plan->units = (plan->blocks + 1) / 2;
    plan->rows = plan->pair ? 2 * kPrefixRows : plan->block_streams * heads;
    // tiles are counted in 32 bits
    const int64_t tiles = (int64_t)(c.n_streams / stream_group) * c.n_kv_heads * plan->units * (c.capacity / kPrefixTile + 1);
    return tiles < 0x7FFFFFFF - 2 * kAttendMaxCtas;
}

cudaError_t launch_prefix(const PrefixParams& p, const void* q, int64_t q_stride, int32_t n_streams, const void* k,
                          const void* v, cudaStream_t st) {
    TraceRange trace("sirllm:attend_shared prefix");
    DeviceProps dp;
    cudaError_t e = device_props(&dp);
    if (e != cudaSuccess) return e;
    EncodeTiled encode;
    if ((e = encoder(&encode)) != cudaSuccess) return e;
    const CUtensorMapDataType type = p.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    CUtensorMap map_q, map_k, map_v;
    {
        const cuuint64_t dims[4] = {(cuuint64_t)p.head_dim, (cuuint64_t)p.heads, (cuuint64_t)p.n_kv_heads, (cuuint64_t)n_streams};
        const cuuint64_t strides[3] = {(cuuint64_t)p.head_dim * 2, (cuuint64_t)p.heads * p.head_dim * 2, (cuuint64_t)q_stride * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)p.heads, 1, (cuuint32_t)p.plan.block_streams};
        if (encode(&map_q, type, 4, const_cast<void*>(q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    for (int i = 0; i < 2; ++i) {
        const cuuint64_t dims[3] = {(cuuint64_t)p.head_dim, (cuuint64_t)p.capacity, (cuuint64_t)n_streams * p.planes_per_stream};
        const cuuint64_t strides[2] = {(cuuint64_t)p.head_dim * 2, (cuuint64_t)p.capacity * p.head_dim * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)kPrefixTile, 1};
        if (encode(i == 0 ? &map_k : &map_v, type, 3, const_cast<void*>(i == 0 ? k : v), dims, strides, box, ones,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    PrefixParams x = p;
    x.q_box_bytes = p.plan.block_streams * p.heads * 128;
    if (p.plan.pair)
        return p.bf16 ? launch<true, true>(x, dp, map_q, map_k, map_v, st) : launch<false, true>(x, dp, map_q, map_k, map_v, st);
    return p.bf16 ? launch<true, false>(x, dp, map_q, map_k, map_v, st) : launch<false, false>(x, dp, map_q, map_k, map_v, st);
}

}  // namespace sirllm
