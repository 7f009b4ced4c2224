// The best continuations of every group of beams (one beam per stream):
//     score(s, v) = total_s + z_sv - lse_s,   lse_s = log sum_v exp z_sv
// over the group's streams s and all tokens v, the n_out largest in order.  An ended beam is one
// candidate, with its total.  Equal scores: the lower stream, then the lower token.
//
// The logits are read once and that is the bound: rows * V elements, a few bytes out.  A CTA takes
// a chunk of one row (up to 32 KB, kept in registers), and gives (max, sum exp) and the chunk's n_out
// best logits; the CTA that finishes a group last joins them: lse in fp64, candidates ranked by
// their score in fp64.  Within a row the order of the logits is the order of the scores.
// The n_out best of many values, twice: every thread knows the largest of its own; the n_out-th of
// those is a bound that n_out values reach, so only what reaches it is listed (a little more than n_out)
// and the list is ranked by counting.  A list that overflows (thousands of equal logits) goes to
// n_out rounds of maximum instead: slow, and right.
#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kThreads = kBeamThreads;
constexpr int kWarps = kThreads / 32;
constexpr int kList = 1024;

// log2 e in two parts: the product's bias would show in lse (1.3e-8 of the distance to the maximum)
constexpr float kLog2eHi = 1.4426950216293335f, kLog2eLo = 1.9259629e-8f;

__device__ __forceinline__ float from_key(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k);
}
__device__ __forceinline__ unsigned long long order_key64(double x) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
__device__ __forceinline__ double from_key64(unsigned long long k) {
    return __longlong_as_double((long long)((k >> 63) ? (k ^ 0x8000000000000000ull) : ~k));
}

// the n-th largest of the threads' values (n <= kThreads), the same for all; syncs
template <typename T>
__device__ __forceinline__ T nth_largest(T mine, T* all, T* found, int n) {
    const int tid = threadIdx.x;
    all[tid] = mine;
    __syncthreads();
    int above = 0;
#pragma unroll 8
    for (int i = 0; i < kThreads; ++i) {
        const T x = all[i];
        above += (x > mine) || (x == mine && i < tid);
    }
    if (above == n - 1) *found = mine;
    __syncthreads();
    return *found;
}

struct Found {                // one candidate of a group
    unsigned long long score;  // order key of its fp64 score
    unsigned long long at;     // (row within the group) << 32 | token
    float z;                   // its logit
};
__device__ __forceinline__ bool better(unsigned long long sa, unsigned long long aa, unsigned long long sb,
                                       unsigned long long ab) {
    return sa > sb || (sa == sb && aa < ab);
}

// kVecs 16-byte vectors of a row per thread
template <bool kBf16, int kVecs>
__global__ void __launch_bounds__(kThreads) beam_kernel(const BeamParams p) {
    constexpr int kPer = kBf16 ? 8 : 4;  // elements of a vector
    __shared__ __align__(16) uint32_t maxima[kThreads];
    __shared__ uint32_t bound;
    __shared__ float warp_m[kWarps];
    __shared__ float warp_s[kWarps];
    __shared__ int listed, last_one;
    __shared__ unsigned long long list[kList];
    __shared__ unsigned long long best[kBeamMaxOut];
    __shared__ unsigned long long warp_best[kWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_dependency_wait();
    grid_launch_dependents();
    const int row = blockIdx.x / p.parts, part = blockIdx.x - row * p.parts;
    const int g = row / p.group;
    const float total = p.totals[row];
    const bool has_ended = p.ended != nullptr && p.ended[row] != 0;

    if (total > -INFINITY && !has_ended) {
        // ---- the chunk, as aligned vectors; what lies outside the row counts as -inf ------------
        const int size = kBf16 ? 2 : 4;
        const char* row_at = static_cast<const char*>(p.logits) + (int64_t)row * p.row_stride * size;
        const int skew = (int)(((uintptr_t)row_at & 15) / size);  // elements in front of the row
        const char* base = row_at - skew * size;
        uint4 raw[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int64_t e0 = ((int64_t)part * kVecs + i) * kThreads * kPer + tid * kPer - skew;  // of the row
            const char* at = base + (e0 + skew) * size;
            if (e0 >= 0 && e0 + kPer <= p.vocab) {
                asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(raw[i].x), "=r"(raw[i].y), "=r"(raw[i].z), "=r"(raw[i].w)
                             : "l"(at));
            } else {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (kBf16) {
                        const int64_t a = e0 + 2 * j, b = a + 1;
                        const uint16_t* q = reinterpret_cast<const uint16_t*>(at);
                        w[j] = (a >= 0 && a < p.vocab ? q[2 * j] : 0xFF80u) |
                               ((uint32_t)(b >= 0 && b < p.vocab ? q[2 * j + 1] : 0xFF80u) << 16);
                    } else {
                        const int64_t a = e0 + j;
                        w[j] = a >= 0 && a < p.vocab ? reinterpret_cast<const uint32_t*>(at)[j] : 0xFF800000u;
                    }
                }
                raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        auto value = [&](int i, int j) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
            if (!kBf16) return __uint_as_float(w[j]);
            return __uint_as_float((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16));
        };
        auto token = [&](int i, int j) {
            return (uint32_t)(((int64_t)part * kVecs + i) * kThreads * kPer + tid * kPer - skew + j);
        };
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j) m = fmaxf(m, value(i, j));
        if (tid == 0) listed = 0;
        float top = m;
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
        if (lane == 0) warp_m[warp] = top;
        const uint32_t reach = nth_largest(order_key(__float_as_uint(m)), maxima, &bound, p.n_out);
        top = warp_m[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, warp_m[w]);
        // ---- sum, and the list of what reaches the bound ---------------------------------------
        const bool any = top > -INFINITY;
        float sum = 0.f;
        if (any) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                float part_sum = 0.f;
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const float t = value(i, j) - top;
                    part_sum += ex2_approx(fmaf(t, kLog2eLo, t * kLog2eHi));
                }
                sum += part_sum;
            }
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        if (lane == 0) warp_s[warp] = sum;
        const uint32_t kLowest = order_key(0xFF800000u);  // -inf: no candidate
        if (order_key(__float_as_uint(m)) >= reach && m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const uint32_t key = order_key(__float_as_uint(value(i, j)));
                    if (key >= reach && key > kLowest) {
                        const int at = atomicAdd(&listed, 1);
                        if (at < kList) list[at] = ((unsigned long long)key << 32) | (0xFFFFFFFFu - token(i, j));
                    }
                }
        }
        if (tid < p.n_out) best[tid] = 0;  // no candidate
        __syncthreads();
        const int n = listed;
        if (n <= kList) {
            for (int i = tid; i < n; i += kThreads) {
                const unsigned long long mine = list[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += list[j] > mine;
                if (rank < p.n_out) best[rank] = mine;
            }
        } else {
            unsigned long long below = ~0ull;
            for (int r = 0; r < p.n_out; ++r) {
                unsigned long long mine = 0;
#pragma unroll
                for (int i = 0; i < kVecs; ++i)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const uint32_t key = order_key(__float_as_uint(value(i, j)));
                        const unsigned long long c = ((unsigned long long)key << 32) | (0xFFFFFFFFu - token(i, j));
                        if (key > kLowest && c < below && c > mine) mine = c;
                    }
#pragma unroll
                for (int x = 16; x > 0; x >>= 1) {
                    const unsigned long long o = __shfl_xor_sync(0xFFFFFFFFu, mine, x);
                    if (o > mine) mine = o;
                }
                if (lane == 0) warp_best[warp] = mine;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w)
                    if (warp_best[w] > mine) mine = warp_best[w];
                if (tid == 0) best[r] = mine;
                below = mine;
                __syncthreads();
            }
        }
        __syncthreads();
        if (tid < p.n_out) p.cands[(int64_t)blockIdx.x * p.n_out + tid] = best[tid];
        if (tid == 0) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) s += warp_s[w];
            p.pairs[blockIdx.x] = any ? make_float2(top, s) : make_float2(0.f, 0.f);
        }
    }
    __syncthreads();
    if (tid == 0) {
        int before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(&p.tickets[g]) : "memory");
        last_one = before == p.group * p.parts - 1;
        if (last_one) p.tickets[g] = 0;  // for the next call
    }
    __syncthreads();
    if (!last_one) return;

    // ---- the group's candidates ---------------------------------------------------------------
    // score of a logit: total + ((z - top) - log sum), top the row's maximum: the differences stay exact
    // where a mask of the type's lowest value is all there is.  A row without candidates: total -inf.
    __shared__ double total_of[kBeamMaxGroup], log_of[kBeamMaxGroup];
    __shared__ float top_of[kBeamMaxGroup];
    __shared__ unsigned char ended_row[kBeamMaxGroup];
    __shared__ unsigned long long maxima64[kThreads], bound64;
    __shared__ Found found[kList];
    __shared__ Found chosen[kBeamMaxOut];
    const int row0 = g * p.group;
    for (int r = warp; r < p.group; r += kWarps) {
        const float t = p.totals[row0 + r];
        const bool e = p.ended != nullptr && p.ended[row0 + r] != 0;
        float top = -INFINITY;
        double sum = 0.0;
        if (t > -INFINITY && !e) {
            for (int i = lane; i < p.parts; i += 32) {
                const float2 v = __ldcg(&p.pairs[(int64_t)(row0 + r) * p.parts + i]);
                if (v.y > 0.f) top = fmaxf(top, v.x);
            }
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
            for (int i = lane; i < p.parts; i += 32) {
                const float2 v = __ldcg(&p.pairs[(int64_t)(row0 + r) * p.parts + i]);
                if (v.y > 0.f) sum += (double)v.y * exp((double)v.x - (double)top);
            }
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        }
        if (lane == 0) {
            ended_row[r] = e;
            top_of[r] = top;
            log_of[r] = log(sum);
            total_of[r] = e || top > -INFINITY ? (double)t : -INFINITY;
        }
    }
    if (tid == 0) listed = 0;
    __syncthreads();
    const int per_row = p.parts * p.n_out, n_cands = p.group * per_row;
    // candidate i: its score's key (0: none), place and logit
    auto candidate = [&](int i, Found& f) {
        const int r = i / per_row, c = i - r * per_row;
        f.score = 0;
        const double total = total_of[r];
        if (!(total > -INFINITY)) return;
        if (ended_row[r]) {
            if (c != 0) return;
            f.score = order_key64(total);
            f.at = (unsigned long long)r << 32;
            f.z = 0.f;
            return;
        }
        const unsigned long long key = __ldcg(&p.cands[(int64_t)(row0 + r) * per_row + c]);
        if (key == 0) return;
        f.z = from_key((uint32_t)(key >> 32));
        f.at = ((unsigned long long)r << 32) | (0xFFFFFFFFu - (uint32_t)key);
        f.score = order_key64(total + (((double)f.z - (double)top_of[r]) - log_of[r]));
    };
    unsigned long long mine = 0;
    for (int i = tid; i < n_cands; i += kThreads) {
        Found f;
        candidate(i, f);
        if (f.score > mine) mine = f.score;
    }
    const unsigned long long reach = nth_largest(mine, maxima64, &bound64, p.n_out);
    if (mine >= reach && mine > 0) {
        for (int i = tid; i < n_cands; i += kThreads) {
            Found f;
            candidate(i, f);
            if (f.score == 0 || f.score < reach) continue;
            const int at = atomicAdd(&listed, 1);
            if (at < kList) found[at] = f;
        }
    }
    if (tid < p.n_out) chosen[tid].score = 0;
    __syncthreads();
    const int n = listed;
    if (n <= kList) {
        for (int i = tid; i < n; i += kThreads) {
            const Found f = found[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += better(found[j].score, found[j].at, f.score, f.at);
            if (rank < p.n_out) chosen[rank] = f;
        }
    } else {
        __shared__ Found warp_found[kWarps];
        unsigned long long last_score = ~0ull, last_at = 0;
        for (int r = 0; r < p.n_out; ++r) {
            Found own;
            own.score = 0;
            own.at = ~0ull;
            own.z = 0.f;
            for (int i = tid; i < n_cands; i += kThreads) {
                Found f;
                candidate(i, f);
                if (f.score == 0 || !better(last_score, last_at, f.score, f.at)) continue;
                if (better(f.score, f.at, own.score, own.at)) own = f;
            }
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) {
                Found o;
                o.score = __shfl_xor_sync(0xFFFFFFFFu, own.score, x);
                o.at = __shfl_xor_sync(0xFFFFFFFFu, own.at, x);
                o.z = __shfl_xor_sync(0xFFFFFFFFu, own.z, x);
                if (better(o.score, o.at, own.score, own.at)) own = o;
            }
            if (lane == 0) warp_found[warp] = own;
            __syncthreads();
            for (int w = 0; w < kWarps; ++w)
                if (better(warp_found[w].score, warp_found[w].at, own.score, own.at)) own = warp_found[w];
            if (tid == 0) chosen[r] = own;
            last_score = own.score;
            last_at = own.at;
            __syncthreads();
            if (own.score == 0) break;
        }
    }
    // ---- out: in order, or a stream's best in the stream's own place and the others in the free ones ---
    __shared__ int first_of[kBeamMaxGroup];       // the first candidate of every row
    __shared__ uint32_t placed[2], taken[2];      // candidates with a place of their own, places taken
    if (tid < kBeamMaxGroup) first_of[tid] = kBeamMaxOut;
    if (tid < 2) taken[tid] = 0;
    __syncthreads();
    const Found f = chosen[tid < p.n_out ? tid : 0];
    const bool real = tid < p.n_out && f.score != 0;
    const int r = real ? (int)(f.at >> 32) : -1;
    int place = tid;
    if (p.places) {  // n_out == group
        if (real) atomicMin(&first_of[r], tid);
        __syncthreads();
        const bool first = real && first_of[r] == tid;
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, first);
        if (lane == 0 && warp < 2) placed[warp] = vote;
        if (first) atomicOr(&taken[r >> 5], 1u << (r & 31));
        __syncthreads();
        if (first) {
            place = r;
        } else if (tid < p.n_out) {
            const uint32_t below = ~placed[warp] & ((1u << lane) - 1u);
            int rank = __popc(below) + (warp == 1 ? __popc(~placed[0]) : 0);  // among those without a place
            for (place = 0; place < p.group; ++place)
                if (!((taken[place >> 5] >> (place & 31)) & 1u) && rank-- == 0) break;
        }
    }
    if (tid < p.n_out) {
        const bool was_ended = real && ended_row[r];
        const int token = !real ? -1 : was_ended ? p.end_token : (int)(uint32_t)f.at;
        const int64_t at = (int64_t)g * p.n_out + place;
        p.totals_out[at] = real ? (float)from_key64(f.score) : -INFINITY;
        p.source[at] = real ? row0 + r : -1;
        p.token_ids[at] = token;
        if (p.entropy != nullptr) p.entropy[at] = real && !was_ended ? (float)(log_of[r] - ((double)f.z - (double)top_of[r])) : 0.f;
        if (p.ended_out != nullptr) p.ended_out[at] = real && (was_ended || (p.end_token >= 0 && token == p.end_token));
    }
}

template <bool kBf16>
cudaError_t launch_vecs(const cudaLaunchConfig_t& cfg, const BeamParams& p) {
    switch (p.vecs) {
        case 1: return cudaLaunchKernelEx(&cfg, beam_kernel<kBf16, 1>, p);
        case 2: return cudaLaunchKernelEx(&cfg, beam_kernel<kBf16, 2>, p);
        case 4: return cudaLaunchKernelEx(&cfg, beam_kernel<kBf16, 4>, p);
        default: return cudaLaunchKernelEx(&cfg, beam_kernel<kBf16, 8>, p);
    }
}

}  // namespace

cudaError_t launch_beam(const BeamParams& p, cudaStream_t st) {
    TraceRange trace("sirllm:beam_select");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.n_streams * p.parts));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return p.logits_dtype == SIRLLM_BF16 ? launch_vecs<true>(cfg, p) : launch_vecs<false>(cfg, p);
}

}  // namespace sirllm
