// Token Entropy straight from the hidden states (Section 3.2, with its remark that the score comes
// with the token's generation): the LM head's product z = hidden * weight^T is formed tile by
// tile in tensor memory and every tile is reduced on the spot to one pair per row,
//     m = max of the tile's logits,  s = sum exp(z - m),
// plus the row's target logit where the tile holds it.  The logits never reach memory; the
// pairs feed sirllm_score_pairs and sirllm_step_pairs.
//
// 2 * rows * columns * d operations on the tensor cores against columns * d * 2 bytes of weight:
// many rows are bound by tcgen05, up to about a hundred rows by reading the weight once.  A
// persistent CTA per SM walks output tiles of 128 rows x up to 256 vocabulary columns, rows
// fastest so that the CTAs at work share weight tiles in L2 and the weight leaves HBM once.
// Warp roles: one lane feeds a ring of TMA loads (64 elements of d per stage, 128-byte swizzle),
// one lane issues tcgen05.mma, four warps reduce the finished accumulator - one thread per row,
// no exchange between threads - while the next tile is multiplied into the other half of TMEM.
// Rows behind the end of a batch or of the vocabulary come in as zeros from TMA and are left out
// of the reduction.  With one block of rows the tile width is chosen so that the tiles fill whole
// waves of SMs.  Products and sums are fp32 (the tensor core's accumulator); nothing is rounded to
// 16 bits on the way.
#include <atomic>

#include <cuda.h>

#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kHeadRows = 128;       // rows of a tile (TMEM lanes)
constexpr int kHeadMaxCols = 256;    // vocabulary columns of a tile, a multiple of 32
constexpr int kHeadDepth = 64;       // elements of d per stage: one 128-byte swizzle row
constexpr int kHeadStages = 4;
constexpr int kHeadThreads = 256;
constexpr int kHeadRowBlocks = 4096; // row blocks per launch (the list of blocks with work)
constexpr float kNoLogit = -2.0e38f;  // below any running maximum; times log2 e it is still finite
constexpr int kABytes = kHeadRows * kHeadDepth * 2;
constexpr int kBBytes = kHeadMaxCols * kHeadDepth * 2;
constexpr int kStageBytes = kABytes + kBBytes;
constexpr size_t kHeadSmem = 1024 + (size_t)kHeadStages * kStageBytes;

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
            dst),
        "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y)
        : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Shared-memory operand of tcgen05.mma, K-major rows of 128 bytes with the 128-byte swizzle:
// groups of 8 rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void tmem_load32(float (&v)[32], uint32_t addr) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,"
        "%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// new tokens of a stream that are scored
__device__ __forceinline__ int stream_rows(const HeadParams& p, int64_t s) {
    return p.n_new ? min(p.n_new[s], p.max_new) : p.max_new;
}

__global__ void __launch_bounds__(kHeadThreads, 1)
head_kernel(const HeadParams p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kHeadStages], empty[kHeadStages], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_base;
    __shared__ int n_active;
    __shared__ volatile int gave_up;
    __shared__ unsigned short active[kHeadRowBlocks];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;

    if (tid == 0) {
        for (int i = 0; i < kHeadStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 4);
        }
        mbar_init(&drained, 1);
        mbar_init_fence();
        gave_up = 0;
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)),
                     "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // row blocks with a row to score, in order
    for (int b = warp; b < p.row_blocks; b += kHeadThreads / 32) {
        bool any = false;
        for (int i = lane; i < kHeadRows; i += 32) {
            const int64_t row = p.row0 + (int64_t)b * kHeadRows + i;
            if (row < p.rows) {
                const int64_t s = row / p.max_new;
                any |= (int)(row - s * p.max_new) < stream_rows(p, s);
            }
        }
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
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    const int blocks = n_active;
    const int64_t n_work = (int64_t)blocks * p.n_tiles;
    const int depth_steps = (p.d_model + kHeadDepth - 1) / kHeadDepth;

    // A wait that runs out raises the flag and every role leaves; the others see it or run out too.
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        for (uint32_t i = 0; i < kMbarSpinLimit; ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if (gave_up) return false;
        }
        gave_up = 1;
        return false;
    };

    if (warp == 0) {
        if (lane == 0) {  // loads
            int stage = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            const uint32_t bytes = (uint32_t)(kABytes + p.tile_cols * kHeadDepth * 2);
            bool ok = true;
            for (int64_t w = blockIdx.x; w < n_work && ok; w += gridDim.x) {
                const int row = (int)(p.row0 + (int64_t)active[w % blocks] * kHeadRows);
                const int col = (int)(w / blocks) * p.tile_cols;
                for (int k = 0; k < depth_steps; ++k) {
                    if (!wait(&empty[stage], phase ^ 1u)) {
                        ok = false;
                        break;
                    }
                    const uint32_t a = tiles + stage * kStageBytes;
                    mbar_expect_tx(&full[stage], bytes);
                    tma_load_2d(a, &map_a, k * kHeadDepth, row, &full[stage]);
                    tma_load_2d(a + kABytes, &map_b, k * kHeadDepth, col, &full[stage]);
                    ++issued;
                    if (++stage == kHeadStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (!ok) {  // let what is in flight land before the CTA's shared memory goes
                const int n = issued < kHeadStages ? (int)issued : kHeadStages;
                for (int i = 0; i < n; ++i) {
                    const int64_t at = issued - 1 - i;
                    mbar_wait_bounded(&full[at % kHeadStages], (uint32_t)((at / kHeadStages) & 1), kMbarSpinLimit);
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {  // products
            // D fp32, A and B of the weight's type, both K-major, 128 rows, tile_cols columns
            const uint32_t idesc = (1u << 4) | ((uint32_t)p.bf16 << 7) | ((uint32_t)p.bf16 << 10) |
                                   ((uint32_t)(p.tile_cols >> 3) << 17) | ((uint32_t)(kHeadRows >> 4) << 24);
            int stage = 0, buf = 0;
            uint32_t phase = 0, buf_phase = 0;
            bool ok = true;
            for (int64_t w = blockIdx.x; w < n_work && ok; w += gridDim.x) {
                ok = wait(&acc_empty[buf], buf_phase ^ 1u);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int k = 0; k < depth_steps; ++k) {
                    ok = wait(&full[stage], phase);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = operand_desc(tiles + stage * kStageBytes);
                    const uint64_t b = operand_desc(tiles + stage * kStageBytes + kABytes);
#pragma unroll
                    for (int i = 0; i < kHeadDepth / 16; ++i)  // 32 bytes of the swizzled rows per step
                        mma_f16(tmem + buf * kHeadMaxCols, a + 2 * i, b + 2 * i, idesc, (k | i) != 0);
                    mma_commit(&empty[stage]);
                    if (++stage == kHeadStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (!ok) break;
                mma_commit(&acc_full[buf]);
                buf ^= 1;
                if (buf == 0) buf_phase ^= 1u;
            }
            if (!ok) {  // products still under way read shared memory and write TMEM
                mma_commit(&drained);
                mbar_wait_bounded(&drained, 0, kMbarSpinLimit);
            }
        }
    } else if (warp >= 4) {  // reduction: one thread per row
        int buf = 0;
        uint32_t buf_phase = 0;
        for (int64_t w = blockIdx.x; w < n_work; w += gridDim.x) {
            const int64_t row = p.row0 + (int64_t)active[w % blocks] * kHeadRows + (tid & 127);
            const int tile = (int)(w / blocks);
            const int64_t col = (int64_t)tile * p.tile_cols;
            const int cols = (int)(p.n_cols - col < p.tile_cols ? p.n_cols - col : p.tile_cols);
            bool on = false;
            int64_t want = -1;  // the target's column within this tile, if it has it
            bool elsewhere = true;
            if (row < p.rows) {
                const int64_t s = row / p.max_new;
                on = (int)(row - s * p.max_new) < stream_rows(p, s);
                if (on) {
                    const int64_t at = (int64_t)p.token_ids[row] - p.col0;
                    elsewhere = at < 0 || at >= p.n_cols;
                    want = at - col;
                }
            }
            if (!wait(&acc_full[buf], buf_phase)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + ((uint32_t)(warp & 3) << 21) + buf * kHeadMaxCols;
            // sum of exp(z) so far = sum * 2^ref, ref = m * log2 e rounded once
            float m = kNoLogit, ref = kNoLogit * kLog2e, sum = 0.f, target = 0.f;
            for (int c = 0; c < cols; c += 32) {
                float z[32];
                tmem_load32(z, acc + c);
                if (c + 32 > cols) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c + i >= cols) z[i] = __uint_as_float(0xFF800000u);
                }
                if (want >= c && want < c + 32) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (want == c + i) target = z[i];
                }
                float top = z[0];
#pragma unroll
                for (int i = 1; i < 32; ++i) top = fmaxf(top, z[i]);
                m = fmaxf(top, m);
                const float old = ref;
                ref = m * kLog2e;
                float s0 = sum * ex2_approx(old - ref), s1 = 0.f;
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    s0 += ex2_approx(fmaf(z[i], kLog2e, -ref));
                    s1 += ex2_approx(fmaf(z[i + 1], kLog2e, -ref));
                }
                sum = s0 + s1;
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf]);
            if (on) {
                // a tile whose logits are all -inf counts for nothing: (0, 0)
                p.pairs_out[row * p.pair_stride + tile] = sum == 0.f ? make_float2(0.f, 0.f) : make_float2(m, sum);
                if (want >= 0 && want < cols)
                    p.target_out[row] = target;
                else if (tile == 0 && elsewhere)
                    p.target_out[row] = 0.f;
            }
            buf ^= 1;
            if (buf == 0) buf_phase ^= 1u;
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
    if (tid == 0 && gave_up) atomicOr(p.status, SIRLLM_STATUS_TIMEOUT);
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, looked up once per process (the library does not link against the driver).
cudaError_t encoder(EncodeTiled* out) {
    static std::atomic<void*> known{nullptr};
    void* fn = known.load(std::memory_order_acquire);
    if (fn == nullptr) {
        cudaDriverEntryPointQueryResult found;
        cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return e;
        if (found != cudaDriverEntryPointSuccess || fn == nullptr) return cudaErrorNotSupported;
        known.store(fn, std::memory_order_release);
    }
    *out = reinterpret_cast<EncodeTiled>(fn);
    return cudaSuccess;
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

}  // namespace

int head_tile_cols(int64_t rows, int64_t n_cols) {
    // Several row blocks: the widest tile, which feeds the tensor core with the fewest bytes.
    if (rows > kHeadRows) return kHeadMaxCols;
    // One row block: reading the weight bounds the call, so its columns are dealt out evenly over
    // whole waves of SMs (a B200 has 148; on another count the result stays right).
    constexpr int64_t kSms = 148;
    const int64_t waves = (n_cols + kSms * kHeadMaxCols - 1) / (kSms * kHeadMaxCols);
    const int64_t share = (n_cols + kSms * waves - 1) / (kSms * waves);
    return (int)((share + 31) / 32 * 32);
}

cudaError_t launch_head(const HeadParams& p, const void* hidden, int64_t hidden_stride, const void* weight,
                        int64_t weight_stride, cudaStream_t st) {
    TraceRange trace("sirllm:head_pairs");
    if (p.rows == 0) return cudaSuccess;
    DeviceProps dp;
    cudaError_t e = device_props(&dp);
    if (e != cudaSuccess) return e;
    EncodeTiled encode;
    if ((e = encoder(&encode)) != cudaSuccess) return e;
    static unsigned char allowed[kMaxDevices];
    if ((e = allow_max_dynamic_smem((const void*)head_kernel, dp, allowed)) != cudaSuccess) return e;
    CUtensorMap map_a, map_b;
    if ((e = row_map(encode, &map_a, hidden, p.rows, p.d_model, hidden_stride, kHeadRows, p.bf16)) != cudaSuccess)
        return e;
    if ((e = row_map(encode, &map_b, weight, p.n_cols, p.d_model, weight_stride, p.tile_cols, p.bf16)) != cudaSuccess)
        return e;
    const int64_t all_blocks = (p.rows + kHeadRows - 1) / kHeadRows;
    for (int64_t b = 0; b < all_blocks; b += kHeadRowBlocks) {
        HeadParams q = p;
        q.row0 = b * kHeadRows;
        q.row_blocks = (int32_t)(all_blocks - b < kHeadRowBlocks ? all_blocks - b : kHeadRowBlocks);
        const int64_t work = (int64_t)q.row_blocks * q.n_tiles;
        const unsigned grid = (unsigned)(work < dp.n_sm ? work : dp.n_sm);
        head_kernel<<<grid, kHeadThreads, kHeadSmem, st>>>(q, map_a, map_b);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace sirllm
