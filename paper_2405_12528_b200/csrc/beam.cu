// The best continuations of every group of beams (one beam per stream):
//     score(s, v) = total_s + z_sv - lse_s,   lse_s = log sum_v exp z_sv
// over the group's streams s and all tokens v, the n_out largest in order.  An ended beam is one
// candidate, with its total.  Equal scores: the lower stream, then the lower token.
//
// The logits are read once and that is the bound: rows * V elements, a few bytes out.  A CTA takes
// a chunk of one row (up to 32 KB, kept in registers), and gives (max, sum exp) and the chunk's n_out
// best logits; the CTA that finishes a group last joins them: sums in fp64, candidates ranked by
// their score in fp64.  Within a row the order of the logits is the order of the scores.
// The n_out best of many values, twice: every thread knows the largest of its own.  The k-th largest of
// every warp's, k * warps >= n_out, the least of them over the warps, is a bound that n_out values reach;
// what reaches it is listed (a few times n_out) and the list is ranked by counting.  A list that
// overflows is made again with the n_out-th largest of all threads' as the bound, and if that overflows
// too (thousands of equal logits) the best come out in n_out rounds of maximum: slow, and right.
#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kThreads = kBeamThreads;
constexpr int kWarps = kThreads / 32;
constexpr int kList = 1024;
constexpr int kFewOut = 8;

// log2 e in two parts: the product's bias would show in lse (1.3e-8 of the distance to the maximum)
constexpr float kLog2eHi = 1.4426950216293335f, kLog2eLo = 1.9259629e-8f;

__device__ __forceinline__ float exp_of(float t) { return ex2_approx(fmaf(t, kLog2eLo, t * kLog2eHi)); }
// order keys of numbers: -0 counts as 0
__device__ __forceinline__ uint32_t key_of(float x) { return order_key(__float_as_uint(x + 0.0f)); }
__device__ __forceinline__ float from_key(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k);
}
__device__ __forceinline__ unsigned long long key64_of(double x) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(x + 0.0);
    return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
__device__ __forceinline__ double from_key64(unsigned long long k) {
    return __longlong_as_double((long long)((k >> 63) ? (k ^ 0x8000000000000000ull) : ~k));
}

// A bound that n of the threads' values reach, or the lowest value where too few threads have one
// (`lowest` says that a thread has none); syncs.
__device__ __forceinline__ float reach_by_warps(float mine, float warp_top, float lowest, int n, float (&tops)[kWarps],
                                                float (&bounds)[kWarps], float (&nths)[kWarps], float& top) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) tops[warp] = warp_top;
    __syncthreads();
    int with = 0;
    top = lowest;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        with += tops[w] > lowest;
        top = fmaxf(top, tops[w]);
    }
    // The k-th largest of the warp, k * warps >= n: the least of those is reached by n values.  And the n-th
    // largest of the warp, for small n: the largest of those is, too.
    uint32_t key = key_of(mine), bound = 0, nth = 0;
    if (warp_top > lowest) {
        const int k = (n + with - 1) / with;
#pragma unroll 1
        for (int i = 1; i <= max(k, n <= kFewOut ? n : 0); ++i) {
            const uint32_t high = __reduce_max_sync(0xFFFFFFFFu, key);
            if (i == k) bound = high;
            nth = high;
            const uint32_t who = __ballot_sync(0xFFFFFFFFu, key == high);
            if (lane == __ffs(who) - 1) key = 0;
        }
    }
    // (more than 32 rounds, or lanes without a value, end at or below the lowest)
    if (lane == 0) {
        bounds[warp] = warp_top > lowest ? (bound == 0 ? lowest : from_key(bound)) : __uint_as_float(0x7F800000u);
        nths[warp] = nth == 0 || n > kFewOut ? lowest : from_key(nth);
    }
    __syncthreads();
    float reach = bounds[0], other = nths[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
        reach = fminf(reach, bounds[w]);
        other = fmaxf(other, nths[w]);
    }
    return fmaxf(reach, other);
}
// the n-th largest of the threads' values (n <= kThreads), the same for all; syncs
__device__ __noinline__ float reach_by_threads(float mine, uint32_t* all, uint32_t* found, int n) {
    const int tid = threadIdx.x;
    const uint32_t key = key_of(mine);
    all[tid] = key;
    __syncthreads();
    int above = 0;
    for (int i = 0; i < kThreads; ++i) {
        const uint32_t x = all[i];
        above += (x > key) || (x == key && i < tid);
    }
    if (above == n - 1) *found = key;
    __syncthreads();
    return from_key(*found);
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

// 16 bytes of a row of which some elements lie outside [0, vocab): those count as -inf
template <bool kBf16>
__device__ __noinline__ uint4 edge_vector(const char* at, int64_t e0, int64_t vocab) {
    uint32_t w[4];
    for (int j = 0; j < 4; ++j) {
        if (kBf16) {
            const int64_t a = e0 + 2 * j, b = a + 1;
            const uint16_t* q = reinterpret_cast<const uint16_t*>(at);
            w[j] = (a >= 0 && a < vocab ? q[2 * j] : 0xFF80u) | (uint32_t)(b >= 0 && b < vocab ? q[2 * j + 1] : 0xFF80u) << 16;
        } else {
            const int64_t a = e0 + j;
            w[j] = a >= 0 && a < vocab ? reinterpret_cast<const uint32_t*>(at)[j] : 0xFF800000u;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool kBf16>
__device__ __forceinline__ float largest(const uint4& v) {
    if (kBf16) {
        uint32_t a, b;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
        return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
    }
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}

struct BeamShared {
    uint32_t maxima[kThreads];
    uint32_t bound;
    float tops[kWarps], bounds[kWarps], nths[kWarps], sums[kWarps];
    int listed, last_one;
    unsigned long long list[kList];    // a chunk's candidates; of a group's, the scores ...
    unsigned long long list_at[kList]; // ... the places
    float list_z[kList];               // ... and the logits
    unsigned long long best[kBeamMaxOut];
    unsigned long long warp_best[kWarps];
    Found warp_found[kWarps], chosen[kBeamMaxOut];
    // of a group's rows.  Score of a logit: total + ((z - top) - log sum), top the row's maximum: the
    // differences stay exact where a mask of the type's lowest value is all there is.  A row without
    // candidates has total -inf.
    double total_of[kBeamMaxGroup], log_of[kBeamMaxGroup];
    float top_of[kBeamMaxGroup];
    unsigned char ended_row[kBeamMaxGroup];
    int first_of[kBeamMaxGroup];       // the first candidate of every row
    uint32_t placed[2], taken[2];      // candidates with a place of their own, places taken
};

// What the chunk's list could not hold: from the logits again.
template <bool kBf16>
__device__ __noinline__ void best_of_many(const BeamParams& p, BeamShared& sh, int row, int64_t first, int length, float m) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float lowest = __uint_as_float(0xFF800000u);
    const int begin = first < 0 ? (int)-first : 0, end = (int)min((int64_t)length, p.vocab - first);
    auto logit = [&](int i) {
        const int64_t at = (int64_t)row * p.row_stride + first + i;
        return kBf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p.logits)[at] << 16)
                     : static_cast<const float*>(p.logits)[at];
    };
    auto candidate = [&](float z, int i) { return ((unsigned long long)key_of(z) << 32) | (0xFFFFFFFFu - (uint32_t)(first + i)); };
    __syncthreads();
    if (tid == 0) sh.listed = 0;
    const float reach = reach_by_threads(m, sh.maxima, &sh.bound, p.n_out);
    for (int i = begin + tid; i < end; i += kThreads) {
        const float z = logit(i);
        if (z >= reach && z > lowest) {
            const int n = atomicAdd(&sh.listed, 1);
            if (n < kList) sh.list[n] = candidate(z, i);
        }
    }
    __syncthreads();
    const int n = sh.listed;
    if (n <= kList) {
        for (int i = tid; i < n; i += kThreads) {
            const unsigned long long mine = sh.list[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += sh.list[j] > mine;
            if (rank < p.n_out) sh.best[rank] = mine;
        }
        return;
    }
    unsigned long long below = ~0ull;
    for (int r = 0; r < p.n_out; ++r) {
        unsigned long long mine = 0;
        for (int i = begin + tid; i < end; i += kThreads) {
            const float z = logit(i);
            const unsigned long long c = candidate(z, i);
            if (z > lowest && c < below && c > mine) mine = c;
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) {
            const unsigned long long o = __shfl_xor_sync(0xFFFFFFFFu, mine, x);
            if (o > mine) mine = o;
        }
        if (lane == 0) sh.warp_best[warp] = mine;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w)
            if (sh.warp_best[w] > mine) mine = sh.warp_best[w];
        if (tid == 0) sh.best[r] = mine;
        below = mine;
        __syncthreads();
    }
}

// kVecs 16-byte vectors of a row per thread
template <bool kBf16, int kVecs>
__device__ __forceinline__ void scan_chunk(const BeamParams& p, BeamShared& sh, int row, int part) {
    constexpr int kPer = kBf16 ? 8 : 4;  // elements of a vector
    constexpr int kSize = kBf16 ? 2 : 4;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // ---- the chunk, as aligned vectors; what lies outside the row counts as -inf ------------------
    const char* row_at = static_cast<const char*>(p.logits) + (int64_t)row * p.row_stride * kSize;
    const int skew = (int)(((uintptr_t)row_at & 15) / kSize);  // elements in front of the row
    const int64_t e_first = (int64_t)part * kVecs * kThreads * kPer + tid * kPer - skew;  // this thread's first element
    const char* at = row_at + e_first * kSize;
    uint4 raw[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t e0 = e_first + i * kThreads * kPer;
        if (e0 >= 0 && e0 + kPer <= p.vocab)
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(raw[i].x), "=r"(raw[i].y), "=r"(raw[i].z), "=r"(raw[i].w)
                         : "l"(at + i * kThreads * 16));
        else
            raw[i] = edge_vector<kBf16>(at + i * kThreads * 16, e0, p.vocab);
    }
    const float lowest = __uint_as_float(0xFF800000u);
    float m = lowest;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) m = fmaxf(m, largest<kBf16>(raw[i]));
    if (tid == 0) sh.listed = 0;
    if (tid < kBeamMaxOut) sh.best[tid] = 0;  // no candidate
    float top;
    const float warp_top = from_key(__reduce_max_sync(0xFFFFFFFFu, key_of(m)));
    const float reach = reach_by_warps(m, warp_top, lowest, p.n_out, sh.tops, sh.bounds, sh.nths, top);
    const bool any = top > lowest;
    // element j of vector i, and its token
    auto value = [&](const uint4& v, int j) {
        const uint32_t w = (kBf16 ? j >> 1 : j) == 0 ? v.x : (kBf16 ? j >> 1 : j) == 1 ? v.y : (kBf16 ? j >> 1 : j) == 2 ? v.z : v.w;
        if (!kBf16) return __uint_as_float(w);
        return __uint_as_float((j & 1) ? (w & 0xFFFF0000u) : (w << 16));
    };
    auto candidate = [&](float z, int i, int j) {
        return ((unsigned long long)key_of(z) << 32) | (0xFFFFFFFFu - (uint32_t)(e_first + i * kThreads * kPer + j));
    };
    uint32_t hits = 0;  // vectors that reach it
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const float high = largest<kBf16>(raw[i]);
        hits |= (uint32_t)(high >= reach && high > lowest) << i;
    }
    // One copy of the code for all of them (unrolled, the instructions' way into the cache took 10 us): the
    // few vectors are read again, from L2.
#pragma unroll 1
    for (; hits != 0; hits &= hits - 1) {
        const int i = __ffs(hits) - 1;
        const int64_t e0 = e_first + i * kThreads * kPer;
        uint4 v;
        if (e0 >= 0 && e0 + kPer <= p.vocab)
            v = __ldg(reinterpret_cast<const uint4*>(at + i * kThreads * 16));
        else
            v = edge_vector<kBf16>(at + i * kThreads * 16, e0, p.vocab);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float z = value(v, j);
            if (z >= reach && z > lowest) {
                const int n = atomicAdd(&sh.listed, 1);
                if (n < kList) sh.list[n] = candidate(z, i, j);
            }
        }
    }
    // ---- the sum ------------------------------------------------------------------------------
    uint64_t sum2[2] = {0, 0};
    if (any) {
        const uint64_t minus_top = pack2(-top, -top), hi = pack2(kLog2eHi, kLog2eHi), lo = pack2(kLog2eLo, kLog2eLo);
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int j = 0; j < kPer; j += 2) {
                const uint64_t t = add2(pack2(value(raw[i], j), value(raw[i], j + 1)), minus_top);
                float a, b;
                unpack2(fma2(t, lo, mul2(t, hi)), a, b);
                sum2[(j >> 1) & 1] = add2(sum2[(j >> 1) & 1], pack2(ex2_approx(a), ex2_approx(b)));
            }
    }
    float s0, s1;
    unpack2(add2(sum2[0], sum2[1]), s0, s1);
    float sum = s0 + s1;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
    if (lane == 0) sh.sums[warp] = sum;
    __syncthreads();
    // ---- the chunk's best ----------------------------------------------------------------------
    const int n = sh.listed;
    if (n <= kList) {
        for (int i = tid; i < n; i += kThreads) {
            const unsigned long long mine = sh.list[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) rank += sh.list[j] > mine;
            if (rank < p.n_out) sh.best[rank] = mine;
        }
    } else {
        best_of_many<kBf16>(p, sh, row, (int64_t)part * kVecs * kThreads * kPer - skew, kVecs * kThreads * kPer, m);
    }
    __syncthreads();
    if (tid < p.n_out) p.cands[(int64_t)blockIdx.x * p.n_out + tid] = sh.best[tid];
    if (tid == 0) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += sh.sums[w];
        p.pairs[blockIdx.x] = any ? make_float2(top, s) : make_float2(0.f, 0.f);
    }
}

// the group's candidates, and what comes of them
__device__ __noinline__ void join_group(const BeamParams& p, BeamShared& sh, int g) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row0 = g * p.group;
    for (int r = warp; r < p.group; r += kWarps) {
        const float t = p.totals[row0 + r];
        const bool e = p.ended != nullptr && p.ended[row0 + r] != 0;
        float top = __uint_as_float(0xFF800000u);
        double sum = 0.0;
        if (t > -INFINITY && !e) {
            const float2* pairs = p.pairs + (int64_t)(row0 + r) * p.parts;
            for (int i = lane; i < p.parts; i += 32) {
                const float2 v = __ldcg(&pairs[i]);
                if (v.y > 0.f) {  // (running: a row of more than 32 chunks)
                    const float up = fmaxf(top, v.x);
                    sum = sum * exp_of(top - up) + (double)v.y * exp_of(v.x - up);
                    top = up;
                }
            }
            const float all = from_key(__reduce_max_sync(0xFFFFFFFFu, key_of(top)));
            if (sum > 0.0) sum *= exp_of(top - all);
            top = all;
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        }
        if (lane == 0) {
            sh.ended_row[r] = e;
            sh.top_of[r] = top;
            sh.log_of[r] = log(sum);
            sh.total_of[r] = e || top > -INFINITY ? (double)t : -INFINITY;
        }
    }
    if (tid == 0) sh.listed = 0;
    __syncthreads();
    const int per_row = p.parts * p.n_out, n_cands = p.group * per_row;
    // candidate i: its score's key (0: none), place and logit
    auto candidate = [&](int i, Found& f) {
        const int r = i / per_row, c = i - r * per_row;
        f.score = 0;
        const double total = sh.total_of[r];
        if (!(total > -INFINITY)) return;
        if (sh.ended_row[r]) {
            if (c != 0) return;
            f.score = key64_of(total);
            f.at = (unsigned long long)r << 32;
            f.z = 0.f;
            return;
        }
        const unsigned long long key = __ldcg(&p.cands[(int64_t)(row0 + r) * per_row + c]);
        if (key == 0) return;
        f.z = from_key((uint32_t)(key >> 32));
        f.at = ((unsigned long long)r << 32) | (0xFFFFFFFFu - (uint32_t)key);
        f.score = key64_of(total + (((double)f.z - (double)sh.top_of[r]) - sh.log_of[r]));
    };
    // The bound is taken among scores rounded to fp32 and no lower than its lowest (rounding keeps the
    // order): -inf stands for no candidate.
    const float none = __uint_as_float(0xFF800000u);
    auto rounded = [](unsigned long long score) { return fmaxf((float)from_key64(score), -3.4028235e38f); };
    float mine = none;
#pragma unroll 1
    for (int i = tid; i < n_cands; i += kThreads) {
        Found f;
        candidate(i, f);
        if (f.score != 0) mine = fmaxf(mine, rounded(f.score));
    }
    float top;
    float reach = reach_by_warps(mine, from_key(__reduce_max_sync(0xFFFFFFFFu, key_of(mine))), none, p.n_out, sh.tops,
                                 sh.bounds, sh.nths, top);
    if (tid < p.n_out) sh.chosen[tid].score = 0;
    int n;
#pragma unroll 1
    for (int again = 0;; ++again) {
        if (mine >= reach && mine > none) {
#pragma unroll 1
            for (int i = tid; i < n_cands; i += kThreads) {
                Found f;
                candidate(i, f);
                if (f.score == 0 || rounded(f.score) < reach) continue;
                const int at = atomicAdd(&sh.listed, 1);
                if (at < kList) {
                    sh.list[at] = f.score;
                    sh.list_at[at] = f.at;
                    sh.list_z[at] = f.z;
                }
            }
        }
        __syncthreads();
        n = sh.listed;
        if (n <= kList || again == 1) break;
        __syncthreads();
        if (tid == 0) sh.listed = 0;
        reach = reach_by_threads(mine, sh.maxima, &sh.bound, p.n_out);
    }
    if (n <= kList) {
#pragma unroll 1
        for (int i = tid; i < n; i += kThreads) {
            const unsigned long long score = sh.list[i], at = sh.list_at[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const unsigned long long x = sh.list[j];
                rank += x > score;
                if (x == score) rank += sh.list_at[j] < at;
            }
            if (rank < p.n_out) sh.chosen[rank] = {score, at, sh.list_z[i]};
        }
    } else {
        unsigned long long last_score = ~0ull, last_at = 0;
#pragma unroll 1
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
            for (int x = 16; x > 0; x >>= 1) {
                Found o;
                o.score = __shfl_xor_sync(0xFFFFFFFFu, own.score, x);
                o.at = __shfl_xor_sync(0xFFFFFFFFu, own.at, x);
                o.z = __shfl_xor_sync(0xFFFFFFFFu, own.z, x);
                if (better(o.score, o.at, own.score, own.at)) own = o;
            }
            if (lane == 0) sh.warp_found[warp] = own;
            __syncthreads();
            for (int w = 0; w < kWarps; ++w)
                if (better(sh.warp_found[w].score, sh.warp_found[w].at, own.score, own.at)) own = sh.warp_found[w];
            if (tid == 0) sh.chosen[r] = own;
            last_score = own.score;
            last_at = own.at;
            __syncthreads();
            if (own.score == 0) break;
        }
    }
    if (tid < kBeamMaxGroup) sh.first_of[tid] = kBeamMaxOut;
    if (tid < 2) sh.taken[tid] = 0;
    __syncthreads();
    // ---- out: in order, or a stream's best in the stream's own place and the others in the free ones ---
    const Found f = sh.chosen[tid < p.n_out ? tid : 0];
    const bool real = tid < p.n_out && f.score != 0;
    const int r = real ? (int)(f.at >> 32) : -1;
    int place = tid;
    if (p.places) {  // n_out == group
        if (real) atomicMin(&sh.first_of[r], tid);
        __syncthreads();
        const bool first = real && sh.first_of[r] == tid;
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, first);
        if (lane == 0 && warp < 2) sh.placed[warp] = vote;
        if (first) atomicOr(&sh.taken[r >> 5], 1u << (r & 31));
        __syncthreads();
        if (first) {
            place = r;
        } else if (tid < p.n_out) {
            const uint32_t below = ~sh.placed[warp] & ((1u << lane) - 1u);
            int rank = __popc(below) + (warp == 1 ? __popc(~sh.placed[0]) : 0);  // among those without a place
#pragma unroll 1
            for (place = 0; place < p.group; ++place)
                if (!((sh.taken[place >> 5] >> (place & 31)) & 1u) && rank-- == 0) break;
        }
    }
    if (tid < p.n_out) {
        const bool was_ended = real && sh.ended_row[r];
        const int token = !real ? -1 : was_ended ? p.end_token : (int)(uint32_t)f.at;
        const int64_t at = (int64_t)g * p.n_out + place;
        p.totals_out[at] = real ? (float)from_key64(f.score) : -INFINITY;
        p.source[at] = real ? row0 + r : -1;
        p.token_ids[at] = token;
        if (p.entropy != nullptr)
            p.entropy[at] = real && !was_ended ? (float)(sh.log_of[r] - ((double)f.z - (double)sh.top_of[r])) : 0.f;
        if (p.ended_out != nullptr) p.ended_out[at] = real && (was_ended || (p.end_token >= 0 && token == p.end_token));
    }
}

template <bool kBf16, int kVecs>
__global__ void __launch_bounds__(kThreads, 4) beam_kernel(const BeamParams p) {
    __shared__ BeamShared sh;
    grid_dependency_wait();
    grid_launch_dependents();
    const int row = blockIdx.x / p.parts, part = blockIdx.x - row * p.parts;
    const int g = row / p.group;
    if (p.totals[row] > -INFINITY && !(p.ended != nullptr && p.ended[row] != 0)) scan_chunk<kBf16, kVecs>(p, sh, row, part);
    __syncthreads();
    if (threadIdx.x == 0) {
        int before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(&p.tickets[g]) : "memory");
        sh.last_one = before == p.group * p.parts - 1;
        if (sh.last_one) p.tickets[g] = 0;  // for the next call
    }
    __syncthreads();
    if (sh.last_one) join_group(p, sh, g);
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
