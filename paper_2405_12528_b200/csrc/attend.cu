// Attention of one new token per stream over a layer's planes:
//     z_j = scale * <q, K_j>,   out = sum_j softmax(z)_j V_j,   lse = log sum_j exp z_j,   j < kv_len
// for every query head; heads g*G .. g*G+G-1 share the planes of K/V head g.
//
// A token does 2 multiply-adds per cache element it reads and per head that shares the element,
// so HBM bounds it: every live K and V row has to come in once.  The cache is cut into tiles of
// 16 slots.  How the tiles are dealt out is decided on the device, where the lengths are: all
// tiles of all (stream, K/V head) units in one line and an equal stretch per CTA - whatever the
// lengths are, the CTAs read the same amount, and a unit that spans CTAs leaves partial results
// (max, sum, weighted rows) in the workspace, joined by the CTA that finishes last, by ticket -
// or whole units per CTA, per cluster of CTAs joined through shared memory, or per warp.  Joins
// add in a fixed order, so results do not depend on timing.  Inside a CTA every warp streams its
// own tiles through its own ring of cp.async stages and keeps a running softmax; nothing but the end
// of a unit makes warps wait for one another, and the ring runs ahead across units.
//
// The products run on mma.sync (m16n8k16) with K and V as the LEFT operand: z^T = K q^T puts 16
// slots on the rows and 8 query heads on the columns, out^T = V^T p^T 16 elements on the rows.
// The group of heads that shares a plane is the narrow side (1 to 8 columns, kTiles * 8 with
// larger groups), so a tile costs one pass over K and one over V whatever the group is; tcgen05
// wants 128 rows of queries or 64+ of K per instruction and a round trip through TMEM for the
// probabilities, and has nothing to give where HBM is the bound.
// fp32: scores, running maximum and sum, output sums, the join.  Rounded to 16 bits: the
// probabilities on their way into the second product, and the result.  The probabilities are taken
// relative to a reference; the true maximum stands between 2^0 and 2^8 of it with bf16, between 2^11
// and 2^15 with fp16, which cannot overflow then, and where what underflows (half a step of 2^-24 a
// slot) is below 2^-36 of the maximum: 49152 faint slots beside a dominant one lose 7e-7 of V.
// Results are 2.3e-3 (bf16) and 2.8e-4 (fp16) of their norm from 64 bits, of which the one rounding at the
// end alone makes 1.7e-3 and 2.1e-4.
// Measured, bf16, heads of 128: 64 streams x 32 heads x 900 - 1280 slots 172 us (1.03 of the copy
// rate, part from L2), 16 x 32 heads x 2048 slots 86 us (0.96), one stream x 8 heads x 12287 slots
// 15.9 us (0.49: launch, reading the length and the join are 7 us of it, and 64 SMs read).
// What the ways to deal out the work bring: 64 x 32 heads x 100 slots 41 us by CTAs, 22 by warps; one
// stream x 8 heads x 2048 slots 17 us by equal shares, 9 by clusters; 22 streams of 1 - 1862 slots x
// 32 heads of 64 108 us by CTAs, 45 by equal shares.
#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kKeys = kAttendTileSlots;
// What an SM reads in the time that joining a unit's parts takes, through memory (6 us at the 110 GB/s
// that one SM takes in, and for each part's rows four times their bytes) and within a cluster (2 us), and
// how many SMs at that rate make up HBM's.
constexpr float kJoinBytes = 640 * 1024, kClusterBytes = 220 * 1024;
constexpr float kBusySms = 58.f;
// What the end of a unit costs a CTA (about 2 us), in bytes of its share of HBM, at most kAttendUnitTiles.
constexpr float kUnitBytes = 96 * 1024;
// The same for a single warp (about 0.9 us), and the longest units, in tiles, that are given to one.
constexpr float kSoloBytes = 96 * 1024;
constexpr int kSoloLongest = 32;
constexpr int kMaxCluster = 8;
// Powers of two between the reference of the probabilities and the largest: where it is set, and
// where it has to move.
template <bool kBf16>
constexpr float kSetBelow = kBf16 ? 0.f : 11.f;
template <bool kBf16>
constexpr float kMoveAt = kBf16 ? 8.f : 15.f;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool kBf16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
template <bool kBf16>
__device__ __forceinline__ uint16_t round16(float v) {
    if (kBf16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    return __half_as_ushort(__float2half_rn(v));
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a shared variable of another CTA of the cluster
__device__ __forceinline__ uint32_t of_rank(const void* p, int rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t a) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(a)
                 : "memory");
    return v;
}

// slots of a stream that count, 0 for a length outside the planes
__device__ __forceinline__ int live_slots(const AttendParams& p, int s) {
    const int n = p.kv_len[s];
    return n < 0 || n > p.capacity ? 0 : n;
}

// A CTA's way through the work, segment by segment.  Two ways: along its stretch of the line of
// tiles, or (whole_units) from unit to unit, `step` units apart.
struct Walk {
    int left;       // positions of the stretch from this segment's first on; whole units: 1 until the end
    int unit0;      // line position of the unit's first tile; whole units: the unit's number
    int s, unit;    // stream; unit within the stream (K/V head, block of query heads)
    int len;        // live slots of the stream
    int t0, t1;     // this segment's tiles of the unit
    int step;       // 0: along the line

    __device__ __forceinline__ bool more() const { return left > 0; }
    __device__ __forceinline__ int tiles() const { return (len + kKeys - 1) / kKeys; }
    __device__ __forceinline__ void set_end() {
        const int T = tiles();
        t1 = step == 0 && T - t0 > left ? t0 + left : T;
    }
    // from the unit numbered unit0, the first one with slots, in steps
    __device__ __forceinline__ void find_unit(const AttendParams& p) {
        const int n_units = p.n_streams * p.units;
        left = 0;
        for (; unit0 < n_units; unit0 += step) {
            s = unit0 / p.units;
            unit = unit0 - s * p.units;
            len = live_slots(p, s);
            if (len > 0) {
                left = 1;
                break;
            }
        }
        t0 = 0;
        set_end();
    }
    // `gap`: positions behind a unit's tiles that stand for what its end costs
    __device__ __forceinline__ void next(const AttendParams& p, const int& gap) {
        if (step > 0) {
            unit0 += step;
            find_unit(p);
            return;
        }
        left -= tiles() + gap - t0;
        if (left <= 0) return;
        unit0 += tiles() + gap;
        t0 = 0;
        if (++unit == p.units) {
            unit = 0;
            for (len = 0; len == 0;) {  // positions are left, so a stream with slots follows
                if (++s >= p.n_streams) {  // (unless the lengths changed under the call)
                    left = 0;
                    return;
                }
                len = live_slots(p, s);
            }
        }
        set_end();
    }
};

// kDim: head_dim rounded up to 64, 128 or 256 (the columns behind head_dim are zeros in shared
// memory); kTiles: blocks of 8 query heads that a unit carries.
template <bool kBf16, int kDim, int kTiles, int kWarps, int kStages>
__global__ void __launch_bounds__(kWarps * 32, 1) attend_kernel(const AttendParams p) {
    constexpr int kThreads = kWarps * 32;
    constexpr int kChunks = kDim / 8;               // 16-byte vectors of a row
    constexpr int kTileBytes = kKeys * kDim * 2;    // K or V of one tile
    constexpr int kHeads = kTiles * 8;
    constexpr int kPass = 4;                        // heads whose output sums are merged at a time
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* ring = smem;                                                   // [warp][stage][K, V]
    float* cta_o = reinterpret_cast<float*>(smem + kWarps * kStages * 2 * kTileBytes);  // [head][head_dim]
    float* merge = cta_o + kHeads * kDim;  // [warp][kPass][kDim]
    __shared__ int scan[kWarps];
    __shared__ int longest[kWarps], counted[kWarps], gap_all;
    __shared__ Walk first;
    __shared__ float stat_m[kWarps][kHeads], stat_l[kWarps][kHeads];
    __shared__ float part_w[kHeads];
    __shared__ __align__(8) float2 cta_ml[kHeads];
    __shared__ int last_one;
    __shared__ float4 team_sum[kThreads];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_dependency_wait();
    grid_launch_dependents();

    // ---- the line of tiles, this CTA's stretch of it -------------------------------------
    const int slice = (p.n_streams + kThreads - 1) / kThreads;
    const int s_lo = min(p.n_streams, tid * slice), s_hi = min(p.n_streams, s_lo + slice);
    const float tile_bytes = (float)(kKeys * 4 * p.head_dim);
    const int gap = min((int)(kUnitBytes / tile_bytes), kAttendUnitTiles);
    int mine = 0, live = 0, long_unit = 0;
    for (int s = s_lo; s < s_hi; ++s) {
        const int T = (live_slots(p, s) + kKeys - 1) / kKeys;
        if (T == 0) continue;
        mine += (T + gap) * p.units;
        ++live;
        long_unit = max(long_unit, T);
    }
    long_unit = __reduce_max_sync(0xFFFFFFFFu, long_unit);
    live = __reduce_add_sync(0xFFFFFFFFu, live);
    int before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, before, o);
        if (lane >= o) before += v;
    }
    if (lane == 31) {
        scan[warp] = before;
        longest[warp] = long_unit;
        counted[warp] = live;
    }
    __syncthreads();
    int line = 0, warps_before = 0;  // below 2^31 - kAttendMaxCtas: a call with more is refused
    live = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) warps_before += scan[w];
        line += scan[w];
        live += counted[w];
        long_unit = max(long_unit, longest[w]);
    }
    before += warps_before - mine;  // tiles in front of this thread's streams
    // Four ways to deal out the work.  (1) An equal share of the line per CTA; units that CTAs share
    // are joined through memory.  (2) Whole units in turn to the CTAs: nothing to join, but no
    // balance between units of different length.  (3) As (2) to the clusters, a unit's tiles in turn
    // to the cluster's CTAs, joined through shared memory.  (4) Whole units in turn to the single
    // warps, which then wait for nobody: for many short units.  The estimate is in tiles that the
    // busiest SM takes in (at 110 GB/s alone, 80 GB/s among many): what HBM takes for all of them
    // (1/kBusySms of the tiles), what the busiest has left when the others are done, and what ends
    // a unit.
    const int total = line - live * p.units * gap;  // tiles
    const float part_tiles = 4.f * (float)(min(kHeads, p.group) * p.head_dim * 4) / tile_bytes;
    // (1): a few very long units are cut into fewer parts than there are SMs: with `per` tiles in a
    // part and long_unit / per parts to join, the sum of both is least at the root
    const int per = max((line + (int)gridDim.x - 1) / (int)gridDim.x, max((int)sqrtf((float)long_unit * part_tiles), 1));
    const float hbm = (float)total * (1.f / kBusySms);
    auto estimate = [&](const AttendDeal& d, int log2_size) {
        const float tiles = (float)((long_unit + (1 << log2_size) - 1) >> log2_size);
        return fmaxf(d.units * (tiles * (4.f / 3.f) + gap), hbm + d.units * tiles - (float)total * d.per_busy);
    };
    float least = fmaxf((float)per * (4.f / 3.f), hbm) + kJoinBytes / tile_bytes +
                  (__fdividef((float)long_unit, (float)per) + 1.f) * part_tiles;
    bool whole_units = false;
    int team = 1;  // CTAs that share a unit
    const float alone = estimate(p.alone, 0);
    if (alone <= least) {
        whole_units = true;
        least = alone;
    }
    if (p.cluster > 1) {
        const float together = estimate(p.together, p.cluster_log2) + kClusterBytes / tile_bytes;
        if (together < least) {
            whole_units = true;
            team = p.cluster;
            least = together;
        }
    }
    // What a tile takes a single warp: 0.9 us of latency over the stages of its ring, 0.15 us of work.
    constexpr float kSoloTile = (0.9f / (kStages - 1) + 0.15f) * 110e3f;  // bytes, as above
    const float solo_tiles =
        p.solo_units * ((float)long_unit * fmaxf((float)kWarps, kSoloTile / tile_bytes) + kSoloBytes / tile_bytes);
    // Single warps take units of up to 512 slots.  Up to there they measured faster than the other ways or 6 %
    // slower at worst (streams x heads of 128 x slots: 64 x 32 x 1 - 512 77 -> 57 us, 192 x 32 x 256 162 ->
    // 137, 192 x 32 x 512 242 -> 256).  With longer units the estimate does not tell even lengths, which lose
    // (192 x 32 x 1024 454 -> 498 us; heads of 64, 64 x 32 x 2048 158 -> 174), from ragged ones, which may gain
    // (64 x 32 x 1 - 768 100 -> 78).  Heads above 128, with four warps to a CTA, keep to the other ways: the
    // estimate is too kind there (heads of 256, 64 x 32 x 1 - 2048 351 -> 442 us), though short units would
    // gain (192 x 32 x 64 161 -> 85).
    const bool solo = kWarps == 8 && long_unit <= kSoloLongest && fmaxf(solo_tiles, hbm) < least;
    if (solo) {
        whole_units = true;
        team = 1;
    }
    const int rank = team > 1 ? (int)cluster_rank() : 0;
    // the warp's first tile of a segment and its way to the next
    const int lead = solo ? 0 : rank * kWarps + warp, stride = solo ? 1 : team * kWarps;
    const int r0 = line / per >= (int)blockIdx.x ? (int)blockIdx.x * per : line;  // (no overflow)
    const int r1 = r0 + min(per, line - r0);
    if (tid == 0) gap_all = gap;
    if (solo) {
        // every warp finds its own first unit below
    } else if (whole_units) {
        if (tid == 0) {
            first.step = gridDim.x / team;
            first.unit0 = blockIdx.x / team;
            first.find_unit(p);
        }
    } else if (r0 >= before && r0 < before + mine) {  // exactly one thread, if the stretch is not empty
        int at = before;
        int s = s_lo, len = 0, T = 0;
        for (; s < s_hi; ++s) {
            len = live_slots(p, s);
            T = len > 0 ? (len + kKeys - 1) / kKeys + gap : 0;  // a unit's positions
            if (r0 < at + T * p.units) break;
            at += T * p.units;
        }
        first.step = 0;
        first.left = s < s_hi ? r1 - r0 : 0;
        if (s < s_hi) {
            first.s = s;
            first.len = len;
            first.unit = (r0 - at) / T;
            first.unit0 = at + first.unit * T;
            first.t0 = r0 - first.unit0;
            first.set_end();
            if (first.t0 >= first.tiles()) first.next(p, gap);  // begins behind a unit's last tile
        }
    }
    // streams without slots: nothing to weigh, the result is zero and its log-sum -inf; a length
    // outside the planes is reported and its rows are left alone
    for (int s = blockIdx.x; s < p.n_streams; s += gridDim.x) {
        const int n = p.kv_len[s];
        if (n < 0 || n > p.capacity) {
            if (tid == 0) atomicOr(p.status, SIRLLM_STATUS_OVERFLOW);
        } else if (n == 0) {
            // (a row of up to 2^31 - 1 elements: the index of the step behind it does not fit an int)
            for (uint32_t i = tid; i < (uint32_t)p.n_heads * p.head_dim; i += kThreads)
                p.out[(int64_t)s * p.out_stride + i] = 0;
            if (p.lse != nullptr)
                for (int i = tid; i < p.n_heads; i += kThreads)
                    p.lse[(int64_t)s * p.n_heads + i] = __uint_as_float(0xFF800000u);
        }
    }
    __syncthreads();
    if (!whole_units && r0 >= line) return;

    // ---- the warp's ring ------------------------------------------------------------------
    const uint32_t ring0 = smem_u32(ring) + warp * kStages * 2 * kTileBytes;
    Walk start = first;
    if (solo) {
        start.step = gridDim.x * kWarps;
        start.unit0 = warp * gridDim.x + blockIdx.x;  // over the SMs first
        start.find_unit(p);
    }
    Walk ahead = start;                 // what the loads have reached
    int ahead_tile = ahead.t0 + lead;
    constexpr int kRowsAtOnce = 32 / kChunks;  // rows that one load instruction of the warp covers
    const int chunk = lane % kChunks, row_in = lane / kChunks;
    const bool chunk_on = chunk * 8 < p.head_dim;
    auto load_next = [&](int stage) {  // the warp's next tile, if there is one, into a stage; one group
        while (ahead.more() && ahead_tile >= ahead.t1) {
            ahead.next(p, gap_all);
            ahead_tile = ahead.t0 + lead;
        }
        if (ahead.more()) {
            const int g = ahead.unit / p.blocks;
            const int64_t plane = (int64_t)ahead.s * p.planes_per_stream + p.layer_plane + g;
            const int key0 = ahead_tile * kKeys;
            const int64_t off = ((plane * p.capacity + key0) * p.head_dim + (chunk_on ? chunk * 8 : 0)) * 2;
            const uint32_t dst0 = ring0 + stage * 2 * kTileBytes;
#pragma unroll
            for (int i = 0; i < kKeys / kRowsAtOnce; ++i) {
                const int r = i * kRowsAtOnce + row_in;
                const bool valid = chunk_on && key0 + r < ahead.len;
                const int64_t o = valid ? off + (int64_t)r * p.head_dim * 2 : off;
                const uint32_t d = dst0 + r * (kDim * 2) + ((chunk ^ (r & 7)) << 4);
                cp_async16(d, p.k + o, valid);
                cp_async16(d + kTileBytes, p.v + o, valid);
            }
            ahead_tile += stride;
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) load_next(i);
    int stage = 0;

    // ---- the units ------------------------------------------------------------------------
    const int hc = 2 * (lane & 3);  // this lane's two heads within a block of 8
    for (Walk w = start; w.more(); w.next(p, gap_all)) {
        const int g = w.unit / p.blocks, block = w.unit - g * p.blocks;
        const int head0 = g * p.group + block * kHeads;            // first query head of the unit
        const int heads = min(kHeads, p.group - block * kHeads);   // query heads it really has
        // queries as the right operand: lane holds elements 2(lane%4), +1 (and +8, +9) of head lane/4
        uint32_t qf[kTiles][kDim / 16][2];
        const char* qrow = p.q + ((int64_t)w.s * p.q_stride + (int64_t)head0 * p.head_dim) * 2;
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
            const int h = n * 8 + (lane >> 2);
#pragma unroll
            for (int ks = 0; ks < kDim / 16; ++ks) {
                const int e = ks * 16 + hc;
                const char* src = qrow + ((int64_t)h * p.head_dim + e) * 2;
                qf[n][ks][0] = h < heads && e < p.head_dim ? *reinterpret_cast<const uint32_t*>(src) : 0u;
                qf[n][ks][1] = h < heads && e + 8 < p.head_dim ? *reinterpret_cast<const uint32_t*>(src + 16) : 0u;
            }
        }
        float o[kTiles][kDim / 16][4];
        float m[kTiles][2], l[kTiles][2];  // reference in units of log2, sum of this lane's slots
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
#pragma unroll
            for (int d = 0; d < kDim / 16; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][d][i] = 0.f;
            m[n][0] = m[n][1] = kNegHuge;
            l[n][0] = l[n][1] = 0.f;
        }
        for (int tile = w.t0 + lead; tile < w.t1; tile += stride) {
            cp_wait<kStages - 2>();
            __syncwarp();
            load_next(stage == 0 ? kStages - 1 : stage - 1);  // the stage that was consumed last
            const uint32_t kt = ring0 + stage * 2 * kTileBytes, vt = kt + kTileBytes;
            float z[kTiles][4];
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[n][i] = 0.f;
            {
                const int r = lane & 15;
                const uint32_t base = kt + r * (kDim * 2);
#pragma unroll
                for (int ks = 0; ks < kDim / 16; ++ks) {
                    uint32_t a[4];
                    ldsm4(a, base + (((2 * ks + (lane >> 4)) ^ (r & 7)) << 4));
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) mma16816<kBf16>(z[n], a, qf[n][ks][0], qf[n][ks][1]);
                }
            }
            // z[n][0..1]: slot lane/4, this lane's two heads; z[n][2..3]: slot lane/4 + 8
            const int key = tile * kKeys + (lane >> 2);
            const bool in0 = key < w.len, in1 = key + 8 < w.len;
            bool raise = false;
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[n][i] = (i < 2 ? in0 : in1) ? z[n][i] * p.scale_log2 : __uint_as_float(0xFF800000u);
                    raise |= z[n][i] > m[n][i & 1] + kMoveAt<kBf16>;
                }
            }
            // The reference moves only when a score passes it by more than that; the sums stay exact.
            if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
                for (int n = 0; n < kTiles; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float top = fmaxf(z[n][i], z[n][i + 2]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
                        const float up = fmaxf(m[n][i], top - kSetBelow<kBf16>);
                        const float f = ex2_approx(m[n][i] - up);
                        m[n][i] = up;
                        l[n][i] *= f;
#pragma unroll
                        for (int d = 0; d < kDim / 16; ++d) {
                            o[n][d][i] *= f;
                            o[n][d][i + 2] *= f;
                        }
                    }
            }
            uint32_t pb[kTiles][2];
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) z[n][i] = ex2_approx(z[n][i] - m[n][i & 1]);
                l[n][0] += z[n][0] + z[n][2];
                l[n][1] += z[n][1] + z[n][3];
                pb[n][0] = transpose8x8(pack16<kBf16>(z[n][0], z[n][1]));
                pb[n][1] = transpose8x8(pack16<kBf16>(z[n][2], z[n][3]));
            }
            {
                const int r = (lane & 7) + ((lane >> 4) << 3);
                const uint32_t base = vt + r * (kDim * 2);
#pragma unroll
                for (int d = 0; d < kDim / 16; ++d) {
                    uint32_t a[4];
                    ldsm4_trans(a, base + (((2 * d + ((lane >> 3) & 1)) ^ (r & 7)) << 4));
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) mma16816<kBf16>(o[n][d], a, pb[n][0], pb[n][1]);
                }
            }
            stage = stage == kStages - 1 ? 0 : stage + 1;
        }
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[n][i] += __shfl_xor_sync(0xFFFFFFFFu, l[n][i], x);
        if (solo) {
            // ---- the warp has the whole unit: four heads at a time through its part of the buffer ------
            float* rows = merge + warp * kPass * kDim;
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int h = n * 8 + hc + i;
                    if (lane < 4 && h < heads && p.lse != nullptr)
                        p.lse[(int64_t)w.s * p.n_heads + head0 + h] = (m[n][i] + log2f(l[n][i])) * (float)kLn2;
                }
#pragma unroll
            for (int q = 0; q < kHeads / kPass; ++q) {
                if (q * kPass >= heads) break;
                const int n = q >> 1;
                if (((lane & 3) >> 1) == (q & 1)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float f = 1.0f / l[n][i];
                        float* row = rows + ((hc & 3) + i) * kDim + (lane >> 2);
#pragma unroll
                        for (int d = 0; d < kDim / 16; ++d) {
                            row[d * 16] = o[n][d][i] * f;
                            row[d * 16 + 8] = o[n][d][i + 2] * f;
                        }
                    }
                }
                __syncwarp();
                const int last = min(kPass, heads - q * kPass);
                for (int h = 0; h < last; ++h)
                    for (int e = 2 * lane; e < p.head_dim; e += 64) {
                        const float2 v = *reinterpret_cast<const float2*>(&rows[h * kDim + e]);
                        *reinterpret_cast<uint32_t*>(p.out + (int64_t)w.s * p.out_stride +
                                                     (int64_t)(head0 + q * kPass + h) * p.head_dim + e) =
                            pack16<kBf16>(v.x, v.y);
                    }
                __syncwarp();
            }
            continue;
        }
        // ---- the warps' sums into one ------------------------------------------------------
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (lane < 4) {
                    stat_m[warp][n * 8 + hc + i] = m[n][i];
                    stat_l[warp][n * 8 + hc + i] = l[n][i];
                }
        __syncthreads();
        const bool shared_unit = team > 1;  // with the cluster's other CTAs
        const bool whole = w.t0 == 0 && w.t1 == w.tiles() && !shared_unit;
        const int c_first = whole_units ? 0 : w.unit0 / per;
        const int64_t slot = 2 * (int64_t)blockIdx.x + ((int)blockIdx.x == c_first ? 1 : 0);
        float* part_o = p.part_o + slot * p.part_heads * p.head_dim;
        float2* part_ml = p.part_ml + slot * p.part_heads;
        float top[kTiles][2];
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float t = kNegHuge;
#pragma unroll
                for (int x = 0; x < kWarps; ++x) t = fmaxf(t, stat_m[x][n * 8 + hc + i]);
                top[n][i] = t;
            }
        if (tid < heads) {
            float t = kNegHuge, sum = 0.f;
#pragma unroll
            for (int x = 0; x < kWarps; ++x) t = fmaxf(t, stat_m[x][tid]);
#pragma unroll
            for (int x = 0; x < kWarps; ++x) sum += stat_l[x][tid] * ex2_approx(stat_m[x][tid] - t);
            if (whole) {
                part_w[tid] = 1.0f / sum;
                if (p.lse != nullptr)
                    p.lse[(int64_t)w.s * p.n_heads + head0 + tid] = (t + log2f(sum)) * (float)kLn2;
            } else if (shared_unit) {
                cta_ml[tid] = make_float2(t, sum);
            } else {
                part_ml[tid] = make_float2(t, sum);
            }
        }
#pragma unroll
        for (int q = 0; q < kHeads / kPass; ++q) {
            if (q * kPass >= heads) break;  // heads is the same for the whole CTA
            const int n = q >> 1;           // block of 8; its lower or upper four heads
            if (((lane & 3) >> 1) == (q & 1)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float f = ex2_approx(m[n][i] - top[n][i]);
                    float* row = merge + (warp * kPass + (hc & 3) + i) * kDim + (lane >> 2);
#pragma unroll
                    for (int d = 0; d < kDim / 16; ++d) {
                        row[d * 16] = o[n][d][i] * f;
                        row[d * 16 + 8] = o[n][d][i + 2] * f;
                    }
                }
            }
            __syncthreads();
            for (int x = tid; x < kPass * kDim; x += kThreads) {
                const int h = q * kPass + x / kDim, e = x % kDim;
                if (h >= heads || e >= p.head_dim) continue;
                float sum = 0.f;
#pragma unroll
                for (int y = 0; y < kWarps; ++y) sum += merge[y * kPass * kDim + x];
                if (whole)
                    p.out[(int64_t)w.s * p.out_stride + (int64_t)(head0 + h) * p.head_dim + e] =
                        round16<kBf16>(sum * part_w[h]);
                else if (shared_unit)
                    cta_o[h * p.head_dim + e] = sum;
                else
                    part_o[h * p.head_dim + e] = sum;
            }
            __syncthreads();
        }
        if (whole) continue;
        if (shared_unit) {
            // ---- the cluster's CTAs into one: each writes its share of the unit's outputs --------
            cluster_sync();
            const int quads = p.head_dim >> 2, items = heads * quads;
            const int share = (items + team - 1) / team;
            const int end = min(items, (rank + 1) * share);
            for (int item = rank * share + tid; item < end; item += kThreads) {
                const int h = item / quads, e = (item - h * quads) * 4;
                float2 ml[kMaxCluster];
                float4 v[kMaxCluster];
                float t = kNegHuge;
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c) {
                    if (c >= team) break;
                    ml[c] = ld_cluster2(of_rank(&cta_ml[h], c));
                    v[c] = ld_cluster4(of_rank(&cta_o[h * p.head_dim + e], c));
                    t = fmaxf(t, ml[c].x);
                }
                float sum = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c) {
                    if (c >= team) break;
                    const float f = ex2_approx(ml[c].x - t);
                    sum = fmaf(ml[c].y, f, sum);
                    acc.x = fmaf(v[c].x, f, acc.x);
                    acc.y = fmaf(v[c].y, f, acc.y);
                    acc.z = fmaf(v[c].z, f, acc.z);
                    acc.w = fmaf(v[c].w, f, acc.w);
                }
                const float f = 1.0f / sum;
                *reinterpret_cast<uint2*>(p.out + (int64_t)w.s * p.out_stride + (int64_t)(head0 + h) * p.head_dim + e) =
                    make_uint2(pack16<kBf16>(acc.x * f, acc.y * f), pack16<kBf16>(acc.z * f, acc.w * f));
                if (e == 0 && p.lse != nullptr)
                    p.lse[(int64_t)w.s * p.n_heads + head0 + h] = (t + log2f(sum)) * (float)kLn2;
            }
            cluster_sync();  // the others have read this CTA's sums
            continue;
        }
        // ---- a unit that several CTAs share: the last one to finish joins the parts --------------
        const int c_last = (w.unit0 + w.tiles() - 1) / per, parts = c_last - c_first + 1;
        __syncthreads();
        if (tid == 0) {
            // release: this CTA's part (all threads' stores, ordered by the barrier) before the ticket;
            // acquire: the ticket before the others' parts are read
            int before_me;
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before_me) : "l"(&p.tickets[c_first]) : "memory");
            last_one = before_me == parts - 1;
            if (last_one) p.tickets[c_first] = 0;  // for the next call
        }
        __syncthreads();
        if (!last_one) continue;
        auto slot_of = [&](int i) { return 2 * (int64_t)(c_first + i) + (i == 0 ? 1 : 0); };
        // four elements per thread; threads that are left over share the parts.  The first rows are
        // asked for before the weights are worked out.
        const int quads = p.head_dim >> 2, items = heads * quads;
        const int teams = items < kThreads ? kThreads / items : 1;
        const int mine = teams > 1 ? tid / items : 0;
        auto row_of = [&](int i, int item) {
            const int h = item / quads;
            return __ldcg(reinterpret_cast<const float4*>(
                &p.part_o[(slot_of(i) * p.part_heads + h) * p.head_dim + (item - h * quads) * 4]));
        };
        constexpr int kEarly = 8;
        float4 early[kEarly];
        const int first_item = tid - mine * items;
        const bool early_on = mine < teams && first_item < items;
#pragma unroll
        for (int j = 0; j < kEarly; ++j)
            early[j] = early_on && mine + j * teams < parts ? row_of(mine + j * teams, first_item)
                                                            : make_float4(0.f, 0.f, 0.f, 0.f);
        // a warp per head: the parts' weights relative to the largest reference, and their sum
        float* weight = merge;  // [part][head]
        for (int h = warp; h < heads; h += kWarps) {
            float2 ml[kAttendMaxCtas / 32];
            float t = kNegHuge;
#pragma unroll
            for (int j = 0; j < kAttendMaxCtas / 32; ++j) {
                const int i = j * 32 + lane;
                ml[j] = i < parts ? __ldcg(&p.part_ml[slot_of(i) * p.part_heads + h]) : make_float2(kNegHuge, 0.f);
                t = fmaxf(t, ml[j].x);
            }
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, x));
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < kAttendMaxCtas / 32; ++j) {
                const float f = ex2_approx(ml[j].x - t);
                if (j * 32 + lane < parts) {
                    sum += ml[j].y * f;
                    weight[(j * 32 + lane) * kHeads + h] = f;
                }
            }
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
            if (lane == 0) {
                part_w[h] = 1.0f / sum;
                if (p.lse != nullptr)
                    p.lse[(int64_t)w.s * p.n_heads + head0 + h] = (t + log2f(sum)) * (float)kLn2;
            }
        }
        __syncthreads();
        for (int base = 0; base < items; base += kThreads) {
            const int item = base + first_item;
            const bool busy = mine < teams && item < items;
            const int h = busy ? item / quads : 0, e = busy ? (item - h * quads) * 4 : 0;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](int i, const float4& v) {
                const float f = weight[i * kHeads + h];
                acc.x = fmaf(v.x, f, acc.x);
                acc.y = fmaf(v.y, f, acc.y);
                acc.z = fmaf(v.z, f, acc.z);
                acc.w = fmaf(v.w, f, acc.w);
            };
            if (busy) {
                int i = mine;
                if (base == 0) {
#pragma unroll
                    for (int j = 0; j < kEarly; ++j, i += teams)
                        if (i < parts) add(i, early[j]);
                }
#pragma unroll 8
                for (; i < parts; i += teams) add(i, row_of(i, item));
            }
            if (teams > 1) {
                team_sum[tid] = acc;
                __syncthreads();
                if (busy && mine == 0) {
                    for (int x = 1; x < teams; ++x) {
                        const float4 v = team_sum[x * items + item];
                        acc.x += v.x;
                        acc.y += v.y;
                        acc.z += v.z;
                        acc.w += v.w;
                    }
                }
            }
            if (busy && mine == 0) {
                const float f = part_w[h];
                const uint2 packed = make_uint2(pack16<kBf16>(acc.x * f, acc.y * f), pack16<kBf16>(acc.z * f, acc.w * f));
                *reinterpret_cast<uint2*>(p.out + (int64_t)w.s * p.out_stride + (int64_t)(head0 + h) * p.head_dim + e) =
                    packed;
            }
        }
        __syncthreads();  // the merge buffer and last_one are used again by the next unit
    }
    cp_wait<0>();
}

template <bool kBf16, int kDim, int kTiles, int kWarps, int kStages>
cudaError_t launch(const AttendParams& p, const DeviceProps& dp, cudaStream_t st) {
    static unsigned char allowed[kMaxDevices];
    auto kernel = attend_kernel<kBf16, kDim, kTiles, kWarps, kStages>;
    cudaError_t e = allow_max_dynamic_smem((const void*)kernel, dp, allowed);
    if (e != cudaSuccess) return e;
    // the ring, a CTA's sums, and a buffer that takes [warp][4 heads][kDim] sums or [part][head] weights
    const size_t sums = (size_t)kWarps * 4 * kDim * 4, weights = (size_t)kAttendMaxCtas * kTiles * 8 * 4;
    const size_t smem = (size_t)kWarps * kStages * 2 * kKeys * kDim * 2 + (size_t)kTiles * 8 * kDim * 4 +
                        (sums > weights ? sums : weights);
    // the largest clusters of which the device holds one per unit
    const int64_t n_units = (int64_t)p.n_streams * p.units;
    AttendParams q = p;
    q.cluster = 1;
    int grid = dp.n_sm < kAttendMaxCtas ? dp.n_sm : kAttendMaxCtas;
    static std::atomic<int> held_cache[kMaxDevices][4];
    for (int i = 3; i > 0; --i) {
        const int size = 1 << i;
        if (n_units * size > grid) continue;
        const bool cached = dp.device >= 0 && dp.device < kMaxDevices;
        int held = cached ? held_cache[dp.device][i].load(std::memory_order_acquire) : 0;
        if (held == 0) {
            cudaLaunchConfig_t ask = {};
            ask.gridDim = dim3(grid / size * size);
            ask.blockDim = dim3(kWarps * 32);
            ask.dynamicSmemBytes = smem;
            cudaLaunchAttribute dim[1];
            dim[0].id = cudaLaunchAttributeClusterDimension;
            dim[0].val.clusterDim.x = size;
            dim[0].val.clusterDim.y = dim[0].val.clusterDim.z = 1;
            ask.attrs = dim;
            ask.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&held, kernel, &ask);
            if (e != cudaSuccess) return e;
            if (cached && held > 0) held_cache[dp.device][i].store(held, std::memory_order_release);
        }
        if (n_units <= held) {
            q.cluster = size;
            grid = (held < grid / size ? held : grid / size) * size;
            break;
        }
    }
    // what the kernel's choice needs of these numbers
    auto deal = [&](int size) {
        const int64_t groups = grid / size;
        AttendDeal d;
        d.units = (float)((n_units + groups - 1) / groups);
        d.per_busy = 1.0f / (float)((n_units < groups ? n_units : groups) * size);
        return d;
    };
    q.alone = deal(1);
    q.together = deal(q.cluster);
    q.solo_units = (float)((n_units + (int64_t)grid * kWarps - 1) / ((int64_t)grid * kWarps));
    q.cluster_log2 = q.cluster == 8 ? 3 : q.cluster == 4 ? 2 : q.cluster == 2 ? 1 : 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = q.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = q.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, q);
}

template <bool kBf16>
cudaError_t launch_dim(const AttendParams& p, const DeviceProps& dp, cudaStream_t st) {
    const bool wide = attend_unit_heads(p.group, p.head_dim) == 16;
    if (p.head_dim <= 64)
        return wide ? launch<kBf16, 64, 2, 8, 6>(p, dp, st) : launch<kBf16, 64, 1, 8, 6>(p, dp, st);
    if (p.head_dim <= 128)
        return wide ? launch<kBf16, 128, 2, 8, 3>(p, dp, st) : launch<kBf16, 128, 1, 8, 3>(p, dp, st);
    return launch<kBf16, 256, 1, 4, 3>(p, dp, st);
}

}  // namespace

cudaError_t launch_attend(const AttendParams& p, bool bf16, cudaStream_t st) {
    TraceRange trace("sirllm:attend");
    DeviceProps dp;
    cudaError_t e = device_props(&dp);
    if (e != cudaSuccess) return e;
    return bf16 ? launch_dim<true>(p, dp, st) : launch_dim<false>(p, dp, st);
}

}  // namespace sirllm
