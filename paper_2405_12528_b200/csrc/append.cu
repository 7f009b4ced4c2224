// New tokens into the cache (Section 3.3: positions are assigned by place in the cache, so the
// token that goes into slot p is token p): queries and keys are normalised per head, turned to
// the position of their slot, and the keys and values are written behind the live slots.
//   norm    y_j = x_j * rsqrt(mean_j x_j^2 + eps) * w_j          (only with weights)
//   rotary  pair i of the head times exp(i * p * theta_i),  theta_i = base^(-2i/d)
//
// Bytes are all there is: every element is read once and written once.  A block takes one token's
// row (few tokens: a share of its heads), asks for all of it at once and computes the row's
// angles, the same for every head, one thread per pair, while the vectors are on their way.  A
// head is handled by a team of lanes (d/16 of them, each with the two 16-byte vectors that carry
// eight pairs), so the norm's sum is a few shuffles inside the team.
// Angles are positions of up to tens of thousands times frequencies down from 1: the number of
// TURNS p * theta / 2pi is formed and reduced in fp64 and only the fraction of a turn goes to
// fp32.  The angle in [-pi, pi] is then off by 3.0e-7 at most (the fraction rounded to fp32 9.4e-8, the
// constant 2pi 8.7e-8, their product 1.2e-7), the fast cosine and sine by their documented 2^-21.19
// and 2^-21.41: each carries up to 7.2e-7 wherever the token sits, a seven hundredth of a rounding to
// fp16.  (Measured where a pair cancels, all angles of 49152 positions: 4.3e-7 of the pair's length.)
// Sums, norm and rotation are fp32; each element is rounded once, to the cache's type.
// Measured, 4096 tokens x 48 heads x 128 bf16 (50 MB in, 50 MB out): 20.9 us with norms (0.75 of the
// copy rate), 18.1 us without; 16384 tokens with norms 68.5 us (0.91); one token 2.4 us.  What is
// left at 4096 tokens is the start and the last, partly filled wave of blocks.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kAppendThreads = 128;
constexpr int kAppendTrips = 8;  // trips of a warp, at most: 1 KB of shared memory each
constexpr int kAppendWarps = kAppendThreads / 32;

template <bool kBf16>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
    if (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    const __half2 h = *reinterpret_cast<const __half2*>(&w);
    return __half22float2(h);
}
template <bool kBf16>
__device__ __forceinline__ float element(const void* p, int i) {
    const uint16_t w = static_cast<const uint16_t*>(p)[i];
    return kBf16 ? __uint_as_float((uint32_t)w << 16) : __half2float(__ushort_as_half(w));
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
__device__ __forceinline__ void unpack_vec(const uint4 v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = unpack16<kBf16>(w[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
}
template <bool kBf16>
__device__ __forceinline__ uint4 pack_vec(const float (&f)[8]) {
    return make_uint4(pack16<kBf16>(f[0], f[1]), pack16<kBf16>(f[2], f[3]), pack16<kBf16>(f[4], f[5]),
                      pack16<kBf16>(f[6], f[7]));
}

__device__ __forceinline__ void copy_async(uint4* dst, const uint4* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// kHalf: pairs (row[i], row[i + d/2]), else (row[2i], row[2i+1]); kNorm: queries, keys or both have weights.
template <bool kBf16, bool kHalf, bool kNorm>
__global__ void __launch_bounds__(kAppendThreads, 9) append_kernel(const __grid_constant__ AppendParams p) {
    // Per pair what turns it: (cosine, sine) - or, with norms, the rotation with the weights folded
    // in, for queries and for keys: a' = r * (a * x + b * y), b' = r * (a * z + b * w), r the
    // reciprocal norm.  Pair 8c + j stands at 32j + c, so that the lanes of a team read side by side.
    __shared__ float2 turned[kNorm ? 1 : SIRLLM_MAX_HEAD_DIM / 2];
    __shared__ float4 folded[kNorm ? 2 : 1][kNorm ? SIRLLM_MAX_HEAD_DIM / 2 : 1];
    extern __shared__ uint4 staged[];
    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row = blockIdx.x / p.groups, group = blockIdx.x - row * p.groups;
    const int s = row / p.max_new, t = row - s * p.max_new;
    const int first = p.first_slot[s];
    const int T = p.n_new ? min(p.n_new[s], p.max_new) : p.max_new;
    if (t >= T) return;
    if (first < 0 || first > p.capacity - T) {
        if (t == 0 && group == 0 && tid == 0) atomicOr(p.status, SIRLLM_STATUS_OVERFLOW);
        return;
    }
    const int slot = first + t;

    // a lane's vectors: pairs 8c .. 8c+7 of a head
    const int units = p.head_dim >> 4;  // lanes of a team with work
    const int c = lane & (p.team - 1), teams = 32 / p.team, member = lane / p.team;
    const bool on = c < units;
    const int va = kHalf ? c : 2 * c, vb = kHalf ? c + units : 2 * c + 1;
    // A trip is one head per team; first the queries' trips, then the keys', then the values'.
    const int q_trips = (p.n_heads + teams - 1) / teams, kv_trips = (p.n_kv_heads + teams - 1) / teams;
    const int trip0 = group * p.trips_per_block + warp;
    const int trip_end = min(p.trips, (group + 1) * p.trips_per_block);
    // All of the warp's vectors are asked for at once, into shared memory: a lane reads back what it
    // asked for itself.
    uint4* const box = staged + warp * p.trips_per_warp * 64 + lane;
    uint4* to = box;
    for (int trip = trip0; trip < trip_end; trip += kAppendWarps, to += 64) {
        const bool is_q = trip < q_trips, is_v = trip >= q_trips + kv_trips;
        const int h = (is_q ? trip : is_v ? trip - q_trips - kv_trips : trip - q_trips) * teams + member;
        const char* base = is_q ? p.q : is_v ? p.v_new : p.k_new;
        const int64_t stride = is_q ? p.q_stride : is_v ? p.v_stride : p.k_stride;
        if (on && h < (is_q ? p.n_heads : p.n_kv_heads)) {
            const uint4* src = reinterpret_cast<const uint4*>(base + (row * stride + h * p.head_dim) * 2);
            copy_async(to, &src[va]);
            copy_async(to + 32, &src[vb]);
        } else {
            to[0] = to[32] = make_uint4(0, 0, 0, 0);
        }
    }
    // meanwhile the row's angles, one thread per pair
    for (int i = tid; i < p.head_dim / 2; i += kAppendThreads) {
        const double turns = (double)slot * p.turns[i];
        const float x = 6.283185307f * (float)(turns - rint(turns));  // [-pi, pi]
        const float cosine = __cosf(x), sine = __sinf(x);
        const int at = (i & 7) * 32 + (i >> 3);
        if (!kNorm) {
            turned[at] = make_float2(cosine, sine);
        } else {
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                const void* w = kind == 0 ? p.q_weight : p.k_weight;
                const float w1 = w ? element<kBf16>(w, kHalf ? i : 2 * i) : 1.f;
                const float w2 = w ? element<kBf16>(w, kHalf ? i + p.head_dim / 2 : 2 * i + 1) : 1.f;
                folded[kind][at] = make_float4(w1 * cosine, -(w2 * sine), w1 * sine, w2 * cosine);
            }
        }
    }
    __syncthreads();
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8 && !kNorm; ++j) {
        const float2 v = turned[32 * j + (on ? c : 0)];
        cs[j] = v.x;
        sn[j] = v.y;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    const uint4* from = box;
    for (int trip = trip0; trip < trip_end; trip += kAppendWarps, from += 64) {
        const bool is_q = trip < q_trips, is_v = trip >= q_trips + kv_trips;
        const int h = (is_q ? trip : is_v ? trip - q_trips - kv_trips : trip - q_trips) * teams + member;
        uint4 xa = from[0], xb = from[32];
        if (!is_v) {
            float a[8], b[8];
            unpack_vec<kBf16>(xa, a);
            unpack_vec<kBf16>(xb, b);
            float r = 1.f;
            if (kNorm && (is_q ? p.q_weight : p.k_weight) != nullptr) {
                float sum = 0.f, sum2 = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sum = fmaf(a[j], a[j], sum);
                    sum2 = fmaf(b[j], b[j], sum2);
                }
                sum += sum2;
                for (int o = p.team >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                r = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
            }
            float u[8], v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // pair j: (a[j], b[j]), or two neighbours in a (j < 4) or b
                const float x = kHalf ? a[j] : j < 4 ? a[2 * (j & 3)] : b[2 * (j & 3)];
                const float y = kHalf ? b[j] : j < 4 ? a[2 * (j & 3) + 1] : b[2 * (j & 3) + 1];
                float x2, y2;
                if (kNorm) {
                    const float4 f = folded[is_q ? 0 : 1][32 * j + (on ? c : 0)];
                    x2 = fmaf(x, f.x, y * f.y) * r;
                    y2 = fmaf(x, f.z, y * f.w) * r;
                } else {
                    x2 = fmaf(x, cs[j], -(y * sn[j]));
                    y2 = fmaf(x, sn[j], y * cs[j]);
                }
                if (kHalf) {
                    u[j] = x2;
                    v[j] = y2;
                } else if (j < 4) {
                    u[2 * (j & 3)] = x2;
                    u[2 * (j & 3) + 1] = y2;
                } else {
                    v[2 * (j & 3)] = x2;
                    v[2 * (j & 3) + 1] = y2;
                }
            }
            xa = pack_vec<kBf16>(u);
            xb = pack_vec<kBf16>(v);
        }
        if (on && h < (is_q ? p.n_heads : p.n_kv_heads)) {
            const int64_t plane = (int64_t)s * p.planes_per_stream + p.layer_plane + h;
            char* dst = is_q ? p.q_out + (row * p.q_out_stride + h * p.head_dim) * 2
                             : (is_v ? p.v : p.k) + (plane * p.capacity + slot) * p.head_dim * 2;
            reinterpret_cast<uint4*>(dst)[va] = xa;
            reinterpret_cast<uint4*>(dst)[vb] = xb;
        }
    }
}

template <bool kBf16, bool kHalf>
cudaError_t launch_norm(const cudaLaunchConfig_t& cfg, const AppendParams& p) {
    return p.q_weight != nullptr || p.k_weight != nullptr
               ? cudaLaunchKernelEx(&cfg, append_kernel<kBf16, kHalf, true>, p)
               : cudaLaunchKernelEx(&cfg, append_kernel<kBf16, kHalf, false>, p);
}
template <bool kBf16>
cudaError_t launch_pairing(const cudaLaunchConfig_t& cfg, const AppendParams& p) {
    return p.layout == SIRLLM_ROPE_HALF ? launch_norm<kBf16, true>(cfg, p) : launch_norm<kBf16, false>(cfg, p);
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, bool bf16, cudaStream_t st) {
    TraceRange trace("sirllm:append_kv");
    const int64_t rows = (int64_t)p.n_streams * p.max_new;
    if (rows == 0) return cudaSuccess;
    DeviceProps dp;
    cudaError_t e = device_props(&dp);
    if (e != cudaSuccess) return e;
    AppendParams q = p;
    const int units = p.head_dim / 16;
    q.team = 1;
    while (q.team < units) q.team *= 2;
    const int teams = 32 / q.team;
    q.inv_dim = 1.0f / (float)p.head_dim;
    q.trips = (p.n_heads + teams - 1) / teams + 2 * ((p.n_kv_heads + teams - 1) / teams);
    // Few rows: one trip per warp, so that a single token's heads spread over the device.  Many rows:
    // a block takes a whole row, whose angles it computes once.
    const int most = rows >= (int64_t)dp.n_sm * 2 ? kAppendTrips : 1;
    q.groups = (q.trips + most * kAppendWarps - 1) / (most * kAppendWarps);
    q.trips_per_block = (q.trips + q.groups - 1) / q.groups;
    q.trips_per_warp = (q.trips_per_block + kAppendWarps - 1) / kAppendWarps;
    if (rows * q.groups > 0x7FFFFFFF) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * q.groups));
    cfg.blockDim = dim3(kAppendThreads);
    cfg.dynamicSmemBytes = (size_t)q.trips_per_warp * 1024 * kAppendWarps;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return bf16 ? launch_pairing<true>(cfg, q) : launch_pairing<false>(cfg, q);
}

}  // namespace sirllm
