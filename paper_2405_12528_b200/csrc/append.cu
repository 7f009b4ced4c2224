// New tokens into the cache (Section 3.3: positions are assigned by place in the cache, so the
// token that goes into slot p is token p): queries and keys are normalised per head, turned to
// the position of their slot, and the keys and values are written behind the live slots.
//   norm    y_j = x_j * rsqrt(mean_j x_j^2 + eps) * w_j          (only with weights)
//   rotary  pair i of the head times exp(i * p * theta_i),  theta_i = base^(-2i/d)
//
// Bytes are all there is: every element is read once and written once.  A head is handled by a
// team of lanes (d/16 of them, each holding the two 16-byte vectors that carry eight pairs), so
// the norm's sum is a few shuffles inside the team, and a row's angles (the same for all of its
// heads) are computed once per warp and kept in registers while the warp walks the heads.
// Angles are positions of up to tens of thousands times frequencies down from 1: the number of
// TURNS p * theta / 2pi is formed and reduced in fp64 and only the fraction of a turn goes to
// fp32 (its sine and cosine carry 2^-24 of absolute error wherever the token sits).  Sums,
// norm and rotation are fp32; each element is rounded once, to the cache's type.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kAppendThreads = 128;

template <bool kBf16>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
    if (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    const __half2 h = *reinterpret_cast<const __half2*>(&w);
    return __half22float2(h);
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

template <bool kBf16>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendParams p) {
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * (kAppendThreads >> 5) + (threadIdx.x >> 5);
    const int64_t row = item / p.groups;
    const int group = (int)(item - row * p.groups);
    if (row >= (int64_t)p.n_streams * p.max_new) return;
    const int s = (int)(row / p.max_new);
    const int t = (int)(row - (int64_t)s * p.max_new);
    const int T = p.n_new ? min(p.n_new[s], p.max_new) : p.max_new;
    if (t >= T) return;
    const int first = p.first_slot[s];
    if (first < 0 || first > p.capacity - T) {
        if (t == 0 && group == 0 && lane == 0) atomicOr(p.status, SIRLLM_STATUS_OVERFLOW);
        return;
    }
    const int slot = first + t;

    // a lane's vectors: pairs 8c .. 8c+7 of a head
    const int units = p.head_dim >> 4;  // lanes of a team with work
    const int c = lane & (p.team - 1);
    const bool on = c < units;
    const int va = p.layout == SIRLLM_ROPE_HALF ? c : 2 * c;
    const int vb = p.layout == SIRLLM_ROPE_HALF ? c + units : 2 * c + 1;
    float cs[8], sn[8];
    if (on) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double turns = (double)slot * p.turns[8 * c + j];
            const float frac = (float)(turns - rint(turns));  // [-0.5, 0.5] of a turn
            sincospif(2.0f * frac, &sn[j], &cs[j]);
        }
    }
    const int teams = 32 / p.team;
    const int h_end = min(p.heads_all, (group + 1) * p.heads_per_group);
    for (int h0 = group * p.heads_per_group; h0 < h_end; h0 += teams) {
        // heads 0 .. n_heads-1 are queries, then come the keys, then the values
        const int h = h0 + lane / p.team;
        const bool has = on && h < h_end;
        const bool is_q = h < p.n_heads, is_v = h >= p.n_heads + p.n_kv_heads;
        const int hk = is_v ? h - p.n_heads - p.n_kv_heads : h - p.n_heads;
        const char* src = is_q   ? p.q + (row * p.q_stride + (int64_t)h * p.head_dim) * 2
                          : is_v ? p.v_new + (row * p.v_stride + (int64_t)hk * p.head_dim) * 2
                                 : p.k_new + (row * p.k_stride + (int64_t)hk * p.head_dim) * 2;
        uint4 xa = make_uint4(0, 0, 0, 0), xb = xa;
        if (has) {
            xa = reinterpret_cast<const uint4*>(src)[va];
            xb = reinterpret_cast<const uint4*>(src)[vb];
        }
        const char* w = static_cast<const char*>(is_q ? p.q_weight : p.k_weight);
        float a[8], b[8];
        unpack_vec<kBf16>(xa, a);
        unpack_vec<kBf16>(xb, b);
        if (p.normed) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(a[j], a[j], fmaf(b[j], b[j], sum));
            for (int o = p.team >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            if (has && !is_v && w != nullptr) {
                const float r = rsqrtf(sum / (float)p.head_dim + p.eps);
                float wa[8], wb[8];
                unpack_vec<kBf16>(reinterpret_cast<const uint4*>(w)[va], wa);
                unpack_vec<kBf16>(reinterpret_cast<const uint4*>(w)[vb], wb);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    a[j] = a[j] * r * wa[j];
                    b[j] = b[j] * r * wb[j];
                }
            }
        }
        if (!has) continue;
        if (!is_v) {
            float u[8], v[8];
            if (p.layout == SIRLLM_ROPE_HALF) {  // a holds the pairs' first elements, b their second
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    u[j] = fmaf(a[j], cs[j], -(b[j] * sn[j]));
                    v[j] = fmaf(a[j], sn[j], b[j] * cs[j]);
                }
            } else {  // pairs side by side: four in a, four in b
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u[2 * j] = fmaf(a[2 * j], cs[j], -(a[2 * j + 1] * sn[j]));
                    u[2 * j + 1] = fmaf(a[2 * j], sn[j], a[2 * j + 1] * cs[j]);
                    v[2 * j] = fmaf(b[2 * j], cs[4 + j], -(b[2 * j + 1] * sn[4 + j]));
                    v[2 * j + 1] = fmaf(b[2 * j], sn[4 + j], b[2 * j + 1] * cs[4 + j]);
                }
            }
            xa = pack_vec<kBf16>(u);
            xb = pack_vec<kBf16>(v);
        }
        char* dst;
        if (is_q) {
            dst = p.q_out + (row * p.q_out_stride + (int64_t)h * p.head_dim) * 2;
        } else {
            const int64_t plane = (int64_t)s * p.planes_per_stream + p.layer_plane + hk;
            dst = (is_v ? p.v : p.k) + (plane * p.capacity + slot) * p.head_dim * 2;
        }
        reinterpret_cast<uint4*>(dst)[va] = xa;
        reinterpret_cast<uint4*>(dst)[vb] = xb;
    }
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
    // Few rows: a warp takes one head per team, so that a single token's heads spread over the
    // device.  Many rows: a warp walks more of a row's heads with the same angles.
    const int trips = (p.heads_all + teams - 1) / teams;
    int64_t per_warp = rows * trips / ((int64_t)dp.n_sm * 32);
    if (per_warp < 1) per_warp = 1;
    if (per_warp > trips) per_warp = trips;
    q.heads_per_group = (int32_t)per_warp * teams;
    q.groups = (p.heads_all + q.heads_per_group - 1) / q.heads_per_group;
    const int64_t blocks = (rows * q.groups + (kAppendThreads / 32) - 1) / (kAppendThreads / 32);
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
    if (bf16)
        append_kernel<true><<<(unsigned)blocks, kAppendThreads, 0, st>>>(q);
    else
        append_kernel<false><<<(unsigned)blocks, kAppendThreads, 0, st>>>(q);
    return cudaGetLastError();
}

}  // namespace sirllm
