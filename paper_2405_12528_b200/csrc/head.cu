// Token Entropy straight from the hidden states (Section 3.2, with its remark that the score comes
// with the token's generation): the LM head's product z = hidden * weight^T is formed tile by
// tile in tensor memory and every tile is reduced on the spot to one pair per row,
//     m = max of the tile's logits,  s = sum exp(z - m),
// plus the row's target logit where the tile holds it.  The logits never reach memory; the
// pairs feed sirllm_score_pairs and sirllm_step_pairs.
//
// 2 * rows * columns * d operations on the tensor cores against columns * d * 2 bytes of weight:
// many rows are bound by tcgen05 (and by what feeds it), up to about a hundred rows by reading
// the weight once.  Three forms, all persistent:
//   kCtas = 2  more than 128 rows.  A pair of CTAs (cta_group::2) multiplies 256 rows by up to 256
//              columns; each CTA loads its own 128 rows and half of the columns, so an SM takes in
//              64 bytes per clock of tensor work where a single CTA's 128 x 256 tile needs 96 -
//              more than L2 delivers.  Tiles go rows fastest: the CTAs at work share weight tiles
//              in L2 and the weight leaves HBM once.
//   kCtas = 1  65 to 128 rows.  Every CTA streams an equal range of weight rows past the one block
//              of hidden rows and keeps one running pair per row for its whole range.
//   few rows   up to 64.  As before, but with the operands exchanged: 128 weight rows on the lanes,
//              16 to 64 hidden rows on the columns.  Padding one row to 128 costs no time by itself,
//              but the energy of 128: a decode loop of 64 rows ran into the power cap (1000 W,
//              1.16 GHz) and took 195 us a step where the first ones took 172.
// Warp roles: one lane feeds a ring of TMA loads (128 elements of d per stage, 128-byte swizzle),
// one lane issues tcgen05.mma, eight warps take the accumulators out of TMEM, which holds two
// of them - one is read while the other is multiplied into.
//
// Precision: the tensor core truncates as it adds, a bias that does not average out and grows with the
// number of additions.  So d is cut into chunks of kChunkSteps stages: a chunk is summed in TMEM, the
// chunks in registers with rounded additions (128 columns of one row per thread), and the bias stays
// that of 1024 elements at any d (measured at 1024 to 16384, the same in all three forms): ordinary
// logits run short by 9e-7 of themselves (fp16 1.2e-6), terms of one sign by 2.2e-6 (fp16 6.1e-6, whose products
// have more bits to lose); unchunked it was 4e-6 for ordinary logits at d = 4096.  Scores are 2e-7 to 1e-6 of
// their norm from 64 bits at d = 1000 to 16384; those of plain fp32 products and sums 4e-8 to 1e-6 up to
// 4096, 2.7e-6 at 16384.  Nothing is rounded to 16 bits.
//
// Measured, bf16: 2048 rows x 37888 columns x 4096 in 371 us (1715 TFLOP/s, 1.03 of cuBLAS's measured
// burst), 4096 x 128256 x 4096 back to back 2.8 - 3.1 ms (1.00 - 1.11 of its rate under the power cap).
// 128256 x 4096 in a loop of 400 calls: 1 row 157 us (6.7 TB/s, 1.04 of the copy rate), 64 rows 164 us (0.99;
// 174 with the board at its power cap), 65 185 us, 100 188 us, 128 201 us, 129 236 us, 256 260 us.
// 32000 x 4096: 1 row 44.5 us (0.91), 64 46.9, 65 48.6, 100 50.4, 129 58.0, 256 60.1.
#include "tcgen05.cuh"

namespace sirllm {

namespace {

constexpr int kHeadRows = 128;       // rows of a CTA (TMEM lanes)
constexpr int kHeadMaxCols = 256;    // vocabulary columns of a tile, at most
constexpr int kHeadDepth = 64;       // elements of d per TMA box: one 128-byte swizzle row
constexpr int kBoxes = 2;            // boxes of A and of B per stage
constexpr int kHeadMaxStages = 8;
// Stages summed in TMEM before they are added up in registers: 1024 elements of d (512 measured 3 %
// slower with many rows, 256 10 % slower with one).
constexpr int kChunkSteps = 8;
constexpr int kHeadReducers = 256;   // threads that reduce: two per row, half of the columns each
constexpr int kHeadThreads = 128 + kHeadReducers;
// Registers: 168 a thread at launch (64512 for 384 threads).  The reducers hold 128 sums each; the
// four warps in front of them hand over what they do not need: 128 * 72 + 256 * 216 = 64512.
constexpr int kFeedRegs = 72, kReduceRegs = 216;
static_assert(128 * kFeedRegs + kHeadReducers * kReduceRegs <= kHeadThreads * 168, "more registers than the launch has");
constexpr int kHeadRowBlocks = 4096; // row blocks per launch (the list of blocks with work)
constexpr int kARoom = kHeadRows * kHeadDepth * 2;  // what an instruction reads of A, loaded or not
constexpr int kHeadRing = 212 * 1024;
constexpr size_t kHeadSmem = 1024 + kHeadRing;
constexpr float kNoLogit = -2.0e38f;  // below any running maximum; times log2 e it is still finite

template <int kCtas>
__device__ __forceinline__ void cta_or_pair_sync() {
    if (kCtas == 2)
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else
        __syncthreads();
}

// a / max_new for 0 <= a < 2^31: multiplication by the rounded-up reciprocal (Granlund and Montgomery)
__device__ __forceinline__ int stream_of(const HeadParams& p, int a) {
    const uint32_t t = __umulhi(p.div_mul, (uint32_t)a);
    return (int)((t + (((uint32_t)a - t) >> p.div_shift1)) >> p.div_shift2);
}
// whether a row holds a token to score: t < n_new[s]
__device__ __forceinline__ bool row_scored(const HeadParams& p, int row) {
    if (row >= p.rows) return false;
    if (p.n_new == nullptr) return true;
    const int s = stream_of(p, row);
    return row - s * p.max_new < p.n_new[s];
}

// A CTA's (or pair's) way through the work: row blocks fastest, then parts.
struct Work {
    int block, part;             // index into the list of active blocks; part
    int blocks, block_step, part_step, parts;
    __device__ __forceinline__ Work(int first, int step, int blocks, int parts) : blocks(blocks), parts(parts) {
        const int n = blocks > 0 ? blocks : 1;
        part = blocks > 0 ? first / n : parts;
        block = first - first / n * n;
        part_step = step / n;
        block_step = step - part_step * n;
    }
    __device__ __forceinline__ bool more() const { return part < parts; }
    __device__ __forceinline__ void next() {
        part += part_step;
        block += block_step;
        if (block >= blocks) {
            block -= blocks;
            ++part;
        }
    }
};

template <int kCtas>
__global__ void __launch_bounds__(kHeadThreads, 1)
head_kernel(const HeadParams p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kHeadMaxStages], empty[kHeadMaxStages], acc_full[2], acc_empty[2], drained;
    __shared__ float4 other_half[2][kHeadRows];
    __shared__ uint32_t tmem_base;
    __shared__ int n_active;
    __shared__ volatile int gave_up;
    __shared__ unsigned short active[kHeadRowBlocks];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = kCtas == 2 ? (int)(blockIdx.x & 1) : 0;  // a cluster is two consecutive CTAs
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
    constexpr int kBlockRows = kHeadRows * kCtas;

    if (tid == 0) {
        for (int i = 0; i < kHeadMaxStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], kCtas * kHeadReducers / 32);
        }
        mbar_init(&drained, 1);
        mbar_init_fence();
        gave_up = 0;
    }
    if (warp == 1) tmem_alloc<kCtas>(&tmem_base);
    // Everything above overlaps the end of the kernel before; from here on its results are read.
    // (Dependents are not released early: CTAs of the next kernel that take an SM's last room while
    // this one drains set the CTAs of the call after it out of step, which cost 8-25 %.)
    grid_dependency_wait();
    // row blocks with a row to score, in order (a single block is not looked at: without a row to
    // score nothing is written)
    for (int b = warp; b < p.row_blocks; b += kHeadThreads / 32) {
        bool any = p.row_blocks == 1;
        for (int i = lane; i < kBlockRows && p.row_blocks > 1; i += 32) any |= row_scored(p, p.row0 + b * kBlockRows + i);
        any = __any_sync(0xFFFFFFFFu, any);
        if (lane == 0) active[b] = any;
    }
    __syncthreads();
    if (warp == 0) {
        int n = 0;
        for (int b0 = 0; b0 < p.row_blocks; b0 += 32) {
            const bool on = b0 + lane < p.row_blocks && active[b0 + lane];
            const uint32_t vote = __ballot_sync(0xFFFFFFFFu, on);
            if (on) active[n + __popc(vote & ((1u << lane) - 1u))] = (unsigned short)(b0 + lane);
            __syncwarp();
            n += __popc(vote);
        }
        if (lane == 0) n_active = n;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cta_or_pair_sync<kCtas>();  // the pair's barriers are set up before either CTA signals them
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    const int blocks = n_active;
    const Work work(blockIdx.x / kCtas, gridDim.x / kCtas, blocks, p.n_parts);
    const int steps = (p.d_model + kBoxes * kHeadDepth - 1) / (kBoxes * kHeadDepth);
    const int chunks = (steps + kChunkSteps - 1) / kChunkSteps;
    // tiles of a part that hold a column
    auto tiles_of = [&](int part) {
        return min(p.part_tiles, p.n_tiles - part * p.part_tiles);
    };

    // A wait that runs out raises the flag and every role leaves; the others see it or run out too.
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        for (uint32_t i = 0; i < kNapLimit; ++i) {
            if (mbar_nap(bar, parity)) return true;
            if (gave_up) return false;
        }
        gave_up = 1;
        return false;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFeedRegs));
        // The loops of these two roles are run by whole warps, so that counters and descriptors stay
        // in uniform registers; one lane issues.  A single thread's instructions are what the tensor
        // core waits for: 64 elements of d (4 instructions) per barrier left it idle 40 % of the
        // time, hence stages of two boxes.
        const bool issuer = lane == 0;
        if (warp == 0) {  // loads
            int issued = 0;
            auto feed = [&]() -> bool {
                int stage = 0;
                uint32_t phase = 0;
                for (Work w = work; w.more(); w.next()) {
                    const int row = p.row0 + active[w.block] * kBlockRows + rank * kHeadRows;
                    const int part = w.part, n_tiles = tiles_of(part);
                    for (int t = 0; t < n_tiles; ++t) {
                        const int col = (part * p.part_tiles + t) * p.tile_cols + rank * (p.tile_cols / kCtas);
                        for (int k = 0; k < steps; ++k) {
                            if (!wait(&empty[stage], phase ^ 1u)) return false;
                            if (issuer) {
                                const uint32_t a = tiles + stage * p.stage_bytes, b = a + kBoxes * p.a_bytes;
                                const uint32_t bar = kCtas == 2 ? in_first_cta(&full[stage]) : smem_u32(&full[stage]);
                                if (rank == 0) mbar_expect_tx(&full[stage], p.load_bytes * kCtas);
#pragma unroll
                                for (int i = 0; i < kBoxes; ++i) {
                                    tma_load_2d<kCtas>(a + i * p.a_bytes, &map_a, (k * kBoxes + i) * kHeadDepth, row, bar);
                                    tma_load_2d<kCtas>(b + i * p.b_bytes, &map_b, (k * kBoxes + i) * kHeadDepth, col, bar);
                                }
                            }
                            if (issued < p.stages) ++issued;
                            if (++stage == p.stages) {
                                stage = 0;
                                phase ^= 1u;
                            }
                        }
                    }
                }
                // leave only when every stage was consumed (and, in a pair, this CTA was told so)
                for (int i = 0; i < p.stages; ++i) {
                    if (!wait(&empty[stage], phase ^ 1u)) return false;
                    if (++stage == p.stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                return true;
            };
            if (!feed() && issuer && rank == 0) {  // gave up: let the loads in flight land
                for (int i = 0; i < issued; ++i)
                    for (uint32_t parity = 0; parity < 2; ++parity) mbar_wait_bounded(&full[i], parity, 1u << 14);
            }
        } else if (warp == 1) {
            auto multiply = [&]() {  // products, for both CTAs of a pair
                // D fp32, A and B of the weight's type, both K-major
                const uint32_t idesc = (1u << 4) | ((uint32_t)p.bf16 << 7) | ((uint32_t)p.bf16 << 10) |
                                       ((uint32_t)(p.tile_cols >> 3) << 17) | ((uint32_t)(kBlockRows >> 4) << 24);
                const uint32_t a_first = operand_lo(tiles), b_first = operand_lo(tiles + kBoxes * p.a_bytes);
                const uint32_t a_box = p.a_bytes >> 4, b_box = p.b_bytes >> 4, next = p.stage_bytes >> 4;
                int stage = 0, buf = 0;
                uint32_t phase = 0, buf_phase = 0, at = 0;
                for (Work w = work; w.more(); w.next()) {
                    const int n_chunks = tiles_of(w.part) * chunks;
                    int left = steps;
                    for (int c = 0; c < n_chunks; ++c) {
                        if (!wait(&acc_empty[buf], buf_phase ^ 1u)) return;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t acc = tmem + buf * kHeadMaxCols;
                        const int n = min(left, kChunkSteps);
                        left = left == n ? steps : left - n;
                        for (int k = 0; k < n; ++k) {
                            if (!wait(&full[stage], phase)) return;
                            if (issuer) {
#pragma unroll
                                for (int i = 0; i < kBoxes; ++i)
#pragma unroll
                                    for (int j = 0; j < kHeadDepth / 16; ++j)  // 32 bytes of the swizzled rows each
                                        mma_f16<kCtas>(acc, a_first + at + i * a_box + 2 * j,
                                                       b_first + at + i * b_box + 2 * j, idesc, (k | i | j) != 0);
                                mma_commit<kCtas>(&empty[stage]);
                            }
                            at += next;
                            if (++stage == p.stages) {
                                stage = 0;
                                at = 0;
                                phase ^= 1u;
                            }
                        }
                        if (issuer) mma_commit<kCtas>(&acc_full[buf]);
                        buf ^= 1;
                        if (buf == 0) buf_phase ^= 1u;
                    }
                }
            };
            if (rank == 0) {
                multiply();
                if (issuer) mma_commit<kCtas>(&drained);
            }
        }
    } else {  // sums of the chunks, then the reduction: a thread has half of a tile's columns of one row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kReduceRegs));
        const int quarter = warp & 3;               // the TMEM lanes a warp may read
        const int half = (warp - 4) >> 2;
        const int r = quarter * 32 + lane;
        const int col_first = half == 0 ? 0 : p.half_cols;
        const int width = half == 0 ? p.half_cols : p.tile_cols - p.half_cols;
        const uint32_t lanes = tmem + ((uint32_t)quarter << 21) + col_first;
        int buf = 0, turn = 0;
        uint32_t buf_phase = 0;
        bool ok = true;
        // What the row of a piece of work is about: asked for a piece ahead, and only looked at when
        // that piece's turn comes.
        struct Row {
            int row, t, n_new, id;
        };
        auto row_of = [&](const Work& w) {
            Row x = {0, 0, 0, -1};
            if (w.more()) {
                x.row = p.row0 + active[w.block] * kBlockRows + rank * kHeadRows + r;
                if (x.row < p.rows) {
                    const int s = stream_of(p, x.row);
                    x.t = x.row - s * p.max_new;
                    x.n_new = p.n_new ? p.n_new[s] : p.max_new;
                    x.id = p.token_ids[x.row];
                }
            }
            return x;
        };
        Work ahead = work;
        Row next = row_of(ahead);
        for (Work w = work; w.more(); w.next()) {
            const int row = next.row, part = w.part;
            const int n_tiles = tiles_of(part);
            const bool on = next.t < next.n_new;              // a row to score
            const bool any = __any_sync(0xFFFFFFFFu, on);     // else this warp's lanes are left alone
            const int64_t at = (int64_t)next.id - p.col0;     // its target's column, if within the range
            ahead.next();
            next = row_of(ahead);
            // sum of exp(z) so far = sum * 2^ref, ref = m * log2 e rounded once
            float m = kNoLogit, ref = kNoLogit * kLog2e, sum = 0.f;
            for (int t = 0; t < n_tiles && ok; ++t) {
                // Always 128 columns: what stands behind a narrower tile's is read and left out below.
                float z[kHeadMaxCols / 2];
#pragma unroll
                for (int i = 0; i < kHeadMaxCols / 2; ++i) z[i] = 0.f;
                for (int c = 0; c < chunks; ++c) {
                    ok = __all_sync(0xFFFFFFFFu, wait(&acc_full[buf], buf_phase));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (any) {
#pragma unroll
                        for (int j = 0; j < kHeadMaxCols / 32; ++j) {
                            float v[16];
                            tmem_load16(v, lanes + buf * kHeadMaxCols + j * 16);
#pragma unroll
                            for (int i = 0; i < 16; ++i) z[j * 16 + i] += v[i];
                        }
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive_cluster(kCtas == 2 ? in_first_cta(&acc_empty[buf]) : smem_u32(&acc_empty[buf]));
                    buf ^= 1;
                    if (buf == 0) buf_phase ^= 1u;
                }
                if (!ok) break;
                if (!any) continue;
                const int64_t col = ((int64_t)part * p.part_tiles + t) * p.tile_cols + col_first;
                const int cols = (int)max((int64_t)0, min((int64_t)width, p.n_cols - col));
                if (cols < kHeadMaxCols / 2) {
#pragma unroll
                    for (int i = 0; i < kHeadMaxCols / 2; ++i)
                        if (i >= cols) z[i] = __uint_as_float(0xFF800000u);
                }
                if (on && at >= col && at < col + cols) {
                    const int want = (int)(at - col);
                    float target = 0.f;
#pragma unroll
                    for (int i = 0; i < kHeadMaxCols / 2; ++i)
                        if (i == want) target = z[i];
                    p.target_out[row] = target;
                }
                float top[4] = {m, m, m, m};  // four chains each: a thread is alone with its row
#pragma unroll
                for (int i = 0; i < kHeadMaxCols / 2; ++i) top[i & 3] = fmaxf(top[i & 3], z[i]);
                m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                const float old = ref;
                ref = m * kLog2e;
                float s[4] = {sum * ex2_approx(old - ref), 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < kHeadMaxCols / 2; ++i) s[i & 3] += ex2_approx(fmaf(z[i], kLog2e, -ref));
                sum = (s[0] + s[1]) + (s[2] + s[3]);
            }
            // the row's two halves into one pair (warps that gave up still meet the others here)
            if (half == 1) other_half[turn][r] = make_float4(m, ref, sum, 0.f);
            asm volatile("bar.sync 1, %0;" ::"n"(kHeadReducers) : "memory");
            if (half == 0 && on && ok) {
                const float4 o = other_half[turn][r];
                const float top = fmaxf(m, o.x), base = top * kLog2e;
                const float s = sum * ex2_approx(ref - base) + o.z * ex2_approx(o.y - base);
                // a part whose logits are all -inf counts for nothing: (0, 0)
                p.pairs_out[(int64_t)row * p.pair_stride + part] = s == 0.f ? make_float2(0.f, 0.f) : make_float2(top, s);
                if (part == 0 && (at < 0 || at >= p.n_cols)) p.target_out[row] = 0.f;  // the token is elsewhere
            }
            turn ^= 1;
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    // Products still under way use both CTAs' shared memory and TMEM.  Waited for here, where every
    // role of this CTA is done and they are due at once: the bound is for one step, not for the call.
    if (warp == 1) {
        if (lane == 0) {
            bool done = false;
            for (uint32_t i = 0; i < kNapLimit && !done; ++i) done = mbar_nap(&drained, 0);
            if (!done) gave_up = 1;
        }
        __syncwarp();
    }
    cta_or_pair_sync<kCtas>();  // neither CTA's memory goes while the other may still use it
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) tmem_free<kCtas>(tmem);
    if (tid == 0 && gave_up) atomicOr(p.status, SIRLLM_STATUS_TIMEOUT);
}

__device__ __forceinline__ void tmem_load8(float (&v)[8], uint32_t addr) {
    uint32_t r[8];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

// Up to kFewRows rows: z^T = weight * hidden^T, 128 vocabulary columns on the lanes and p.few_cols
// (16, 32, 48 or 64) rows on the columns of an accumulator.  A reducing thread keeps the running
// pairs of half of the rows over its lane's columns of the whole part; the 128 lanes are joined once,
// at the part's end, by shuffles.  The last tile of a part loads only the columns that the part has
// left (map_t); what else its lanes multiply is not looked at.
constexpr int kFewRows = 64;
constexpr int64_t kFewShare = 32;  // columns of a part, at least
__global__ void __launch_bounds__(kHeadThreads, 1)
head_few_kernel(const HeadParams p, const __grid_constant__ CUtensorMap map_h, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_t) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kHeadMaxStages], empty[kHeadMaxStages], acc_full[2], acc_empty[2], drained;
    __shared__ float2 quarters[4][kFewRows];  // a row's pair over 32 lanes
    __shared__ int want[kFewRows];            // a row's target column within the part, -1 if elsewhere
    __shared__ int scored[kFewRows];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int gave_up;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
    constexpr int kTile = kHeadRows;          // vocabulary columns of a tile

    if (tid == 0) {
        for (int i = 0; i < kHeadMaxStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], kHeadReducers / 32);
        }
        mbar_init(&drained, 1);
        mbar_init_fence();
        gave_up = 0;
    }
    if (warp == 1) tmem_alloc<1>(&tmem_base);
    grid_dependency_wait();  // as in head_kernel
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    const int steps = (p.d_model + kBoxes * kHeadDepth - 1) / (kBoxes * kHeadDepth);
    const int chunks = (steps + kChunkSteps - 1) / kChunkSteps;

    // A wait that runs out raises the flag and every role leaves; the others see it or run out too.
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        for (uint32_t i = 0; i < kNapLimit; ++i) {
            if (mbar_nap(bar, parity)) return true;
            if (gave_up) return false;
        }
        gave_up = 1;
        return false;
    };

    if (warp == 0) {
        const bool issuer = lane == 0;
        int issued = 0;
        auto feed = [&]() -> bool {
            int stage = 0;
            uint32_t phase = 0;
            for (int part = blockIdx.x; part < p.n_parts; part += gridDim.x) {
                for (int t = 0; t < p.part_tiles; ++t) {
                    const bool tail = t == p.part_tiles - 1;
                    const int col = part * p.part_cols + t * kTile;
                    const uint32_t bytes = p.load_bytes - (tail ? kBoxes * (kTile - p.tail_cols) * kHeadDepth * 2 : 0);
                    for (int k = 0; k < steps; ++k) {
                        if (!wait(&empty[stage], phase ^ 1u)) return false;
                        if (issuer) {
                            const uint32_t a = tiles + stage * p.stage_bytes, b = a + kBoxes * kARoom;
                            mbar_expect_tx(&full[stage], bytes);
#pragma unroll
                            for (int i = 0; i < kBoxes; ++i) {
                                const int depth = (k * kBoxes + i) * kHeadDepth;
                                tma_load_2d<1>(a + i * kARoom, tail ? &map_t : &map_w, depth, col, smem_u32(&full[stage]));
                                tma_load_2d<1>(b + i * p.b_bytes, &map_h, depth, 0, smem_u32(&full[stage]));
                            }
                        }
                        if (issued < p.stages) ++issued;
                        if (++stage == p.stages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                }
            }
            return true;
        };
        if (!feed() && issuer) {  // gave up: let the loads in flight land
            for (int i = 0; i < issued; ++i)
                for (uint32_t parity = 0; parity < 2; ++parity) mbar_wait_bounded(&full[i], parity, 1u << 14);
        }
    } else if (warp == 1) {
        const bool issuer = lane == 0;
        auto multiply = [&]() {
            const uint32_t idesc = (1u << 4) | ((uint32_t)p.bf16 << 7) | ((uint32_t)p.bf16 << 10) |
                                   ((uint32_t)(p.few_cols >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
            const uint32_t a_first = operand_lo(tiles), b_first = operand_lo(tiles + kBoxes * kARoom);
            const uint32_t b_box = p.b_bytes >> 4, next = p.stage_bytes >> 4;
            int stage = 0, buf = 0;
            uint32_t phase = 0, buf_phase = 0, at = 0;
            for (int part = blockIdx.x; part < p.n_parts; part += gridDim.x) {
                int left = steps;
                for (int c = 0; c < p.part_tiles * chunks; ++c) {
                    if (!wait(&acc_empty[buf], buf_phase ^ 1u)) return;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t acc = tmem + buf * kFewRows;
                    const int n = min(left, kChunkSteps);
                    left = left == n ? steps : left - n;
                    for (int k = 0; k < n; ++k) {
                        if (!wait(&full[stage], phase)) return;
                        if (issuer) {
#pragma unroll
                            for (int i = 0; i < kBoxes; ++i)
#pragma unroll
                                for (int j = 0; j < kHeadDepth / 16; ++j)
                                    mma_f16<1>(acc, a_first + at + i * (kARoom >> 4) + 2 * j,
                                               b_first + at + i * b_box + 2 * j, idesc, (k | i | j) != 0);
                            mma_commit<1>(&empty[stage]);
                        }
                        at += next;
                        if (++stage == p.stages) {
                            stage = 0;
                            at = 0;
                            phase ^= 1u;
                        }
                    }
                    if (issuer) mma_commit<1>(&acc_full[buf]);
                    buf ^= 1;
                    if (buf == 0) buf_phase ^= 1u;
                }
            }
        };
        multiply();
        if (issuer) {
            mma_commit<1>(&drained);  // products still under way use shared memory and TMEM
            if (!mbar_wait_bounded(&drained, 0, kMbarSpinLimit)) gave_up = 1;
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, half = (warp - 4) >> 2, me = tid - 128;
        const int r = quarter * 32 + lane;                   // the tile's column of this lane
        const int mine = p.few_cols >> 1, base = half * mine;  // this thread's rows
        const uint32_t lanes = tmem + ((uint32_t)quarter << 21) + base;
        int buf = 0;
        uint32_t buf_phase = 0;
        bool ok = true;
        for (int part = blockIdx.x; part < p.n_parts; part += gridDim.x) {
            const int64_t first = (int64_t)part * p.part_cols;
            if (me < kFewRows) {
                bool on = false;
                int64_t at = -1;
                if (row_scored(p, me)) {
                    on = true;
                    at = (int64_t)p.token_ids[me] - p.col0;
                    if (part == 0 && (at < 0 || at >= p.n_cols)) p.target_out[me] = 0.f;  // the token is elsewhere
                    if (at >= p.n_cols) at = -1;
                    at = at >= first && at < first + p.part_cols ? at - first : -1;
                }
                scored[me] = on;
                want[me] = (int)at;
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kHeadReducers) : "memory");
            float m[kFewRows / 2], s[kFewRows / 2];
#pragma unroll
            for (int i = 0; i < kFewRows / 2; ++i) {
                m[i] = kNoLogit;
                s[i] = 0.f;
            }
            for (int t = 0; t < p.part_tiles && ok; ++t) {
                float z[kFewRows / 2];
#pragma unroll
                for (int i = 0; i < kFewRows / 2; ++i) z[i] = 0.f;
                for (int c = 0; c < chunks; ++c) {
                    if (!(ok = __all_sync(0xFFFFFFFFu, wait(&acc_full[buf], buf_phase)))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int j = 0; j < kFewRows / 16; ++j) {
                        if (j * 8 < mine) {
                            float v[8];
                            tmem_load8(v, lanes + buf * kFewRows + j * 8);
#pragma unroll
                            for (int i = 0; i < 8; ++i) z[j * 8 + i] += v[i];
                        }
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(smem_u32(&acc_empty[buf]));
                    buf ^= 1;
                    if (buf == 0) buf_phase ^= 1u;
                }
                if (!ok) break;
                // rows whose target is one of this tile's columns: the lane that has it writes it
                const int at = lane < mine ? want[base + lane] - t * kTile : -1;
                for (uint32_t hit = __ballot_sync(0xFFFFFFFFu, at >= 0 && at < kTile && want[base + lane] >= 0); hit != 0;
                     hit &= hit - 1) {
                    const int i = __ffs(hit) - 1;
                    if (__shfl_sync(0xFFFFFFFFu, at, i) == r) {
                        float target = 0.f;
#pragma unroll
                        for (int x = 0; x < kFewRows / 2; ++x)
                            if (x == i) target = z[x];
                        p.target_out[base + i] = target;
                    }
                }
                const int cols = t == p.part_tiles - 1 ? p.tail_cols : kTile;
                if (r < cols && first + t * kTile + r < p.n_cols) {
#pragma unroll
                    for (int j = 0; j < kFewRows / 16; ++j) {
                        if (j * 8 < mine) {
#pragma unroll
                            for (int x = 0; x < 8; ++x) {
                                const int i = j * 8 + x;
                                const float top = fmaxf(m[i], z[i]);
                                const float f = ex2_approx((fminf(m[i], z[i]) - top) * kLog2e);
                                s[i] = z[i] > m[i] ? fmaf(s[i], f, 1.f) : s[i] + f;
                                m[i] = top;
                            }
                        }
                    }
                }
            }
            // 32 lanes into one, then the four quarters
#pragma unroll
            for (int j = 0; j < kFewRows / 16; ++j) {
                if (j * 8 < mine) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const int i = j * 8 + x;
                        float top = m[i];
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                        float sum = s[i] * ex2_approx((m[i] - top) * kLog2e);
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                        if (lane == x) quarters[quarter][base + i] = make_float2(top, sum);
                    }
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kHeadReducers) : "memory");
            if (me < p.few_cols && scored[me] && ok) {
                float top = kNoLogit, sum = 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q) top = fmaxf(top, quarters[q][me].x);
#pragma unroll
                for (int q = 0; q < 4; ++q) sum += quarters[q][me].y * ex2_approx((quarters[q][me].x - top) * kLog2e);
                // a part whose logits are all -inf counts for nothing: (0, 0)
                p.pairs_out[(int64_t)me * p.pair_stride + part] = sum == 0.f ? make_float2(0.f, 0.f) : make_float2(top, sum);
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kHeadReducers) : "memory");  // before the tables are filled again
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) tmem_free<1>(tmem);
    if (tid == 0 && gave_up) atomicOr(p.status, SIRLLM_STATUS_TIMEOUT);
}

// Rows of `width` 16-bit elements, `stride` elements apart, read in boxes of box_rows x 64.
cudaError_t row_map(EncodeTiled encode, CUtensorMap* map, const void* base, int64_t rows, int width, int64_t stride,
                    int box_rows, bool bf16) {
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {(cuuint32_t)kHeadDepth, (cuuint32_t)box_rows};
    const cuuint32_t ones[2] = {1, 1};
    const CUresult r = encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                              const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int kCtas>
cudaError_t launch(const HeadParams& p, unsigned grid, const DeviceProps& dp, const CUtensorMap& a, const CUtensorMap& b,
                   cudaStream_t st) {
    static unsigned char allowed[kMaxDevices];
    cudaError_t e = allow_max_dynamic_smem((const void*)head_kernel<kCtas>, dp, allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kHeadThreads);
    cfg.dynamicSmemBytes = kHeadSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCtas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kCtas == 2 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, head_kernel<kCtas>, p, a, b);
}

// What a tile costs besides its columns, in columns (the reduction takes 128 a thread, used or not).
constexpr int64_t kTileEnd = 64;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What stream_of multiplies and shifts by.
void division(HeadParams* q) {
    const uint32_t d = (uint32_t)q->max_new;
    int l = 0;
    while (((uint64_t)1 << l) < d) ++l;
    q->div_mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1);
    q->div_shift1 = l < 1 ? l : 1;
    q->div_shift2 = l > 0 ? l - 1 : 0;
}

}  // namespace

// The cut depends on the sizes alone (callers size their pairs by it), for the 148 SMs of a B200;
// on another count of SMs the results are the same and only the balance differs.
HeadTiling head_tiling(int64_t rows, int64_t n_cols) {
    constexpr int64_t kSms = 148;
    HeadTiling t;
    if (rows <= kFewRows) {
        // Reading the weight bounds the call, so its columns are dealt out evenly, one range per SM, in
        // tiles of 128 of which the last is loaded as far as it goes.
        t.ctas = 0;
        int64_t share = ceil_div(ceil_div(n_cols, kSms), 8) * 8;
        if (share < kFewShare) share = kFewShare;
        t.part_cols = (int32_t)share;
        t.tile_cols = kHeadRows;
        t.part_tiles = (int32_t)ceil_div(share, kHeadRows);
        t.half_cols = 0;
        t.n_parts = (int32_t)ceil_div(n_cols, share);
        return t;
    }
    if (rows <= kHeadRows) {
        // One block of rows: reading the weight bounds the call, so its columns are dealt out evenly,
        // one range per SM, each cut into equal tiles.
        t.ctas = 1;
        const int64_t share = ceil_div(ceil_div(n_cols, kSms), 16) * 16;
        t.part_tiles = (int32_t)ceil_div(share, kHeadMaxCols);
        t.tile_cols = (int32_t)(ceil_div(ceil_div(share, t.part_tiles), 16) * 16);
        t.half_cols = (int32_t)ceil_div(t.tile_cols / 2, 16) * 16;
    } else {
        // The widest tile feeds the tensor core with the fewest bytes; a narrower one is taken where
        // it shortens the last wave of tiles by more than that costs.
        t.ctas = 2;
        t.part_tiles = 1;
        const int64_t blocks = ceil_div(rows, 2 * kHeadRows);
        int64_t best = 0;
        t.tile_cols = kHeadMaxCols;
        for (int64_t c = kHeadMaxCols; c >= 64; c -= 32) {
            const int64_t cost = ceil_div(blocks * ceil_div(n_cols, c), kSms / 2) * (c + kTileEnd);
            if (best == 0 || cost * 33 < best * 32) {
                best = cost;
                t.tile_cols = (int32_t)c;
            }
        }
        t.half_cols = t.tile_cols / 2;
    }
    t.part_cols = t.part_tiles * t.tile_cols;
    t.n_parts = (int32_t)ceil_div(n_cols, t.part_cols);
    return t;
}

cudaError_t launch_head(const HeadParams& p, const HeadTiling& t, const void* hidden, int64_t hidden_stride,
                        const void* weight, int64_t weight_stride, cudaStream_t st) {
    TraceRange trace("sirllm:head_pairs");
    if (p.rows == 0) return cudaSuccess;
    DeviceProps dp;
    cudaError_t e = device_props(&dp);
    if (e != cudaSuccess) return e;
    EncodeTiled encode;
    if ((e = encoder(&encode)) != cudaSuccess) return e;
    if (t.ctas == 0) {
        HeadParams q = p;
        q.few_cols = (int32_t)ceil_div(p.rows, 16) * 16;
        q.n_parts = t.n_parts;
        q.part_tiles = t.part_tiles;
        q.part_cols = t.part_cols;
        q.tail_cols = t.part_cols - (t.part_tiles - 1) * kHeadRows;
        q.b_bytes = q.few_cols * kHeadDepth * 2;
        q.load_bytes = kBoxes * (kARoom + q.b_bytes);
        q.stage_bytes = q.load_bytes;
        q.stages = kHeadRing / q.stage_bytes;
        if (q.stages > kHeadMaxStages) q.stages = kHeadMaxStages;
        division(&q);
        CUtensorMap map_h, map_w, map_t;
        if ((e = row_map(encode, &map_h, hidden, p.rows, p.d_model, hidden_stride, q.few_cols, p.bf16)) != cudaSuccess ||
            (e = row_map(encode, &map_w, weight, p.n_cols, p.d_model, weight_stride, kHeadRows, p.bf16)) != cudaSuccess ||
            (e = row_map(encode, &map_t, weight, p.n_cols, p.d_model, weight_stride, q.tail_cols, p.bf16)) != cudaSuccess)
            return e;
        static unsigned char few_allowed[kMaxDevices];
        if ((e = allow_max_dynamic_smem((const void*)head_few_kernel, dp, few_allowed)) != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(q.n_parts < dp.n_sm ? q.n_parts : dp.n_sm));
        cfg.blockDim = dim3(kHeadThreads);
        cfg.dynamicSmemBytes = kHeadSmem;
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, head_few_kernel, q, map_h, map_w, map_t);
    }
    const int a_rows = t.ctas == 2 ? kHeadRows : (int)ceil_div(p.rows, 8) * 8;
    const int b_rows = t.tile_cols / t.ctas;
    CUtensorMap map_a, map_b;
    if ((e = row_map(encode, &map_a, hidden, p.rows, p.d_model, hidden_stride, a_rows, p.bf16)) != cudaSuccess) return e;
    if ((e = row_map(encode, &map_b, weight, p.n_cols, p.d_model, weight_stride, b_rows, p.bf16)) != cudaSuccess)
        return e;
    HeadParams q = p;
    q.n_parts = t.n_parts;
    q.n_tiles = (int32_t)ceil_div(p.n_cols, t.tile_cols);
    q.part_tiles = t.part_tiles;
    q.tile_cols = t.tile_cols;
    q.half_cols = t.half_cols;
    // a stage: the rows that are loaded, swizzle groups of 8 rows (1 KB) at a time
    q.a_bytes = a_rows * kHeadDepth * 2;
    q.b_bytes = b_rows * kHeadDepth * 2;
    q.load_bytes = kBoxes * (q.a_bytes + q.b_bytes);
    q.stage_bytes = q.load_bytes;
    // an instruction reads 128 rows of A from a stage's start; the ring leaves room for that at its end
    q.stages = (kHeadRing - (kARoom - q.a_bytes)) / q.stage_bytes;
    if (q.stages > kHeadMaxStages) q.stages = kHeadMaxStages;
    division(&q);
    const int64_t block_rows = (int64_t)kHeadRows * t.ctas;
    const int64_t all_blocks = ceil_div(p.rows, block_rows);
    for (int64_t b = 0; b < all_blocks; b += kHeadRowBlocks) {
        q.row0 = (int32_t)(b * block_rows);
        q.row_blocks = (int32_t)(all_blocks - b < kHeadRowBlocks ? all_blocks - b : kHeadRowBlocks);
        const int64_t work = (int64_t)q.row_blocks * q.n_parts, fit = dp.n_sm / t.ctas;
        const unsigned grid = (unsigned)((work < fit ? work : fit) * t.ctas);
        e = t.ctas == 2 ? launch<2>(q, grid, dp, map_a, map_b, st) : launch<1>(q, grid, dp, map_a, map_b, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace sirllm
