// The best continuations of every group of beams (one beam per stream):
//     score(s, v) = total_s + z_sv - lse_s,   lse_s = log sum_v exp z_sv
// over the group's streams s and all tokens v, the n_out largest in order.  An ended beam is one
// candidate, with its total.  Equal scores: the lower stream, then the lower token.
//
// The logits are read once and that is the bound: rows * V elements, a few bytes out.  A warp streams a
// segment of one row and keeps the running maximum and sum per lane; of every block of 512 bytes it leaves
// the largest logit, and looks for no candidates.  The CTA whose warp finishes a group last joins its
// segments (sums in fp64) and takes the n_out best SEGMENTS of the group, by their largest logit's score
// and then by place: they hold the n_out best candidates, for each of n_out better segments would bring
// a better candidate.  In the same way the n_out best blocks of these, and then the n_out best logits
// of these blocks, the only ones that are read again; the last of the n_out is the bound for the next level.
// Scores are compared in fp64; within a row the order of the logits is the order of the scores.
// A lane's sum is fp32 over up to 64 trips, each at most 6 roundings of 2^-24 (an addition, and an exp and a product where
// the maximum moves); segments are joined in fp64.
// What reaches the bound is listed and ranked by counting.  A list that overflows is made again with the
// n_out-th largest of all threads' best as the bound, and if that overflows too (thousands of equal
// scores) the best come out in n_out rounds of maximum: slow, and right.
// Measured, bf16: 512 rows x 128256 (8 to a group, four fifths of them live) 41.0 us, of which the search takes 15; all of
// them live and off the 16-byte boundaries (128257 wide) 48.1; 128 x 128256, 16 candidates 24.5; 4 x 32000 10.4; 64 beams and
// candidates 40 - 65.  The search waits for loads that depend on one another and for instructions that are executed once.
// On the way here, 512 x 128256 bf16: chunks of 32 KB per CTA, with barriers between loading, bounding,
// listing and ranking, 61 us; warps that keep lists of their own while they stream, 83 us; blocks
// without segments, bounds taken anew at every level, 53 us.  Ranking
// by one 128-bit entry per candidate, eight at a time, in place of three arrays: two groups of 64 beams 73 -> 57 us.
#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kThreads = kBeamThreads;
constexpr int kWarps = kThreads / 32;
constexpr int kList = 1024;
constexpr int kRankStep = 8;  // entries compared with at a time
constexpr int kLevels = 3;
constexpr int kFewBlocks = 2048;
constexpr int kRankAll = 64;
constexpr int kBatch = 8;  // items that a lane asks for at a time
constexpr int kStep = 4;   // vectors of a lane per trip: blocks of a trip
static_assert(kStep * 512 == kBeamTripBytes, "a trip is kStep blocks");

// log2 e in two parts: the product's bias would show in lse (1.3e-8 of the distance to the maximum)
constexpr float kLog2eHi = 1.4426950216293335f, kLog2eLo = 1.9259629e-8f;

__device__ __forceinline__ float exp_of(float t) { return ex2_approx(fmaf(t, kLog2eLo, t * kLog2eHi)); }
constexpr float kLowest = -3.4028235e38f;  // of all numbers
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
                                                float (&bounds)[kWarps], float (&nths)[kWarps]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) tops[warp] = warp_top;
    __syncthreads();
    int with = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) with += tops[w] > lowest;
    // The k-th largest of the warp, k * warps >= n: the least of those is reached by n values.  And the n-th
    // largest of the warp, for small n: the largest of those is, too.
    uint32_t key = key_of(mine), bound = 0, nth = 0;
    if (warp_top > lowest) {
        const int k = (n + with - 1) / with;
#pragma unroll 1
        for (int i = 1; i <= max(k, n <= 32 ? n : 0); ++i) {
            const uint32_t high = __reduce_max_sync(0xFFFFFFFFu, key);
            if (i == k) bound = high;
            nth = high;
            const uint32_t who = __ballot_sync(0xFFFFFFFFu, key == high);
            if (lane == __ffs(who) - 1) key = 0;
        }
    }
    if (with == 0) return lowest;
    // (more than 32 rounds, or lanes without a value, end at or below the lowest)
    if (lane == 0) {
        bounds[warp] = warp_top > lowest ? (bound == 0 ? lowest : from_key(bound)) : __uint_as_float(0x7F800000u);
        nths[warp] = nth == 0 || n > 32 ? lowest : from_key(nth);
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

// One candidate of a group (or segment, or block).  Of equal scores the better one has the lower place: the lower
// stream, then the larger logit (a huge total hides it), then the lower token.
constexpr int kIndexBits = 26;
struct __align__(16) Found {
    unsigned long long score;  // order key of its fp64 score; 0: none
    unsigned long long place;  // row within the group (6 bits), order key of its logit inverted, index
    __device__ __forceinline__ int row() const { return (int)(place >> (32 + kIndexBits)); }
    __device__ __forceinline__ int index() const { return (int)(place & ((1u << kIndexBits) - 1u)); }
    __device__ __forceinline__ float logit() const { return from_key(~(uint32_t)(place >> kIndexBits)); }
};
static_assert(SIRLLM_MAX_BEAMS <= 64 && SIRLLM_MAX_BEAM_VOCAB <= 1 << kIndexBits, "a place fits 64 bits");
__device__ __forceinline__ unsigned long long place_of(int row, float z, int index) {
    return ((unsigned long long)row << (32 + kIndexBits)) | ((unsigned long long)~key_of(z) << kIndexBits) | (uint32_t)index;
}
__device__ __forceinline__ bool better(const Found& a, const Found& b) {
    return a.score > b.score || (a.score == b.score && a.place < b.place);
}

// 16 bytes of a row of which some elements lie outside [0, vocab): those count as -inf
template <bool kBf16>
__device__ __noinline__ uint4 edge_vector(const char* at, int e0, int vocab) {
    uint32_t w[4];
    for (int j = 0; j < 4; ++j) {
        if (kBf16) {
            const int a = e0 + 2 * j, b = a + 1;
            const uint16_t* q = reinterpret_cast<const uint16_t*>(at);
            w[j] = (a >= 0 && a < vocab ? q[2 * j] : 0xFF80u) | (uint32_t)(b >= 0 && b < vocab ? q[2 * j + 1] : 0xFF80u) << 16;
        } else {
            const int a = e0 + j;
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
    Found list[kList + kRankStep];  // what reaches the bound
    uint32_t maxima[kThreads];
    uint32_t bound;
    float tops[kWarps], bounds[kWarps], nths[kWarps];
    int listed;
    Found warp_found[kWarps], chosen[kLevels][kBeamMaxOut];  // the best segments, blocks, candidates
    // of a group's rows.  Score of a logit: total + ((z - top) - log sum), top the row's maximum: the
    // differences stay exact where a mask of the type's lowest value is all there is.  A row without
    // candidates has total -inf.
    double total_of[kBeamMaxGroup], log_of[kBeamMaxGroup];
    float top_of[kBeamMaxGroup], const_of[kBeamMaxGroup];  // const: total - log sum, -inf for a row without logits that count
    __device__ __forceinline__ unsigned long long score(unsigned long long place) const {  // its order key
        const Found f = {0, place};
        const int r = f.row();
        return key64_of(ended_row[r] ? total_of[r]
                                     : total_of[r] + (((double)f.logit() - (double)top_of[r]) - log_of[r]));
    }
    unsigned char ended_row[kBeamMaxGroup];
    int first_of[kBeamMaxGroup];       // the first candidate of every row
    uint32_t placed[2], taken[2];      // candidates with a place of their own, places taken
};

// One warp's segment of a row: p.trips trips of kStep vectors per lane.  Segments, blocks and lanes go by the
// elements' indices, so that equal rows have equal sums wherever they begin (a tie between streams is one then).
// kWords >= 0: the row begins off a 16-byte boundary, so many words and perhaps half a word behind it.  A lane puts
// its vector together from the aligned one that it loads and words of the next lane's; those behind a trip's last
// vector come by a load of lane 31's own.
constexpr int kAligned = -1;
template <bool kBf16, int kWords>
__device__ __forceinline__ void scan_segment(const BeamParams& p, int row, int part) {
    constexpr int kPer = kBf16 ? 8 : 4;  // elements of a vector
    constexpr int kSize = kBf16 ? 2 : 4;
    const int lane = threadIdx.x & 31;
    // as aligned vectors; what lies outside the row counts as -inf
    const char* row_at = static_cast<const char*>(p.logits) + (int64_t)row * p.row_stride * kSize;
    const int skew = kWords == kAligned ? 0 : (int)((uintptr_t)row_at & 15);  // bytes in front of the row
    const int first_block = part * p.trips * kStep;
    const int trips = min(p.trips, (p.blocks - first_block + kStep - 1) / kStep);
    const int vocab = (int)p.vocab;
    int e_next = (first_block * 32 + lane) * kPer - skew / kSize;  // first element of the lane's next vector
    auto load_in = [&](uint4& v, int e0) {
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(row_at + (int64_t)e0 * kSize));
    };
    auto load_one = [&](uint4& v, int e0) {
        if (e0 >= 0 && e0 + kPer <= vocab)
            load_in(v, e0);
        else
            v = edge_vector<kBf16>(row_at + (int64_t)e0 * kSize, e0, vocab);
    };
    // Inside the row there is nothing to check per vector (512 x 128256 bf16 42.7 -> 40.7 us; off the boundaries 50.1 -> 47.9).
    auto load = [&](uint4 (&v)[kStep], uint4& behind) {
        const int e_first = e_next - lane * kPer;
        if (e_first >= 0 && e_first + (kStep * 32 + 1) * kPer <= vocab) {
#pragma unroll
            for (int i = 0; i < kStep; ++i) load_in(v[i], e_next + i * 32 * kPer);
            if (kWords != kAligned && lane == 31) load_in(behind, e_next + ((kStep - 1) * 32 + 1) * kPer);
            e_next += kStep * 32 * kPer;
            return;
        }
#pragma unroll
        for (int i = 0; i < kStep; ++i) load_one(v[i], e_next + i * 32 * kPer);
        if (kWords != kAligned && lane == 31) load_one(behind, e_next + ((kStep - 1) * 32 + 1) * kPer);
        e_next += kStep * 32 * kPer;
    };
    // vector i of a trip: kWords words (and, bf16, perhaps half a word) behind where v[i] begins
    constexpr int kFrom = kWords == kAligned ? 0 : kWords + (kBf16 ? 1 : 0);  // words of the next lane
    const int half = kBf16 ? (skew & 2) * 8 : 0;
    auto word = [](const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; };
    auto assemble = [&](uint4 (&v)[kStep], const uint4& behind) {
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = word(v[i], j);
#pragma unroll
            for (int j = 0; j < kFrom; ++j) {
                const uint32_t give = i + 1 < kStep && lane == 0 ? word(v[(i + 1) % kStep], j) : x[j];
                x[4 + j] = __shfl_sync(0xFFFFFFFFu, give, lane + 1);  // (lane 31 from lane 0)
                if (i + 1 == kStep && lane == 31) x[4 + j] = word(behind, j);
            }
            constexpr int k = kWords == kAligned ? 0 : kWords;
            if (kBf16)
                v[i] = make_uint4(__funnelshift_r(x[k], x[k + 1], half), __funnelshift_r(x[k + 1], x[k + 2], half),
                                  __funnelshift_r(x[k + 2], x[k + 3], half), __funnelshift_r(x[k + 3], x[k + 4], half));
            else
                v[i] = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
        }
    };
    auto value = [&](const uint4& v, int j) {  // element j
        const uint32_t w = (kBf16 ? j >> 1 : j) == 0 ? v.x : (kBf16 ? j >> 1 : j) == 1 ? v.y : (kBf16 ? j >> 1 : j) == 2 ? v.z : v.w;
        if (!kBf16) return __uint_as_float(w);
        return __uint_as_float((j & 1) ? (w & 0xFFFF0000u) : (w << 16));
    };
    float top = kLowest, sum = 0.f;
    float* block_max = p.block_max + (int64_t)row * p.blocks + first_block;
    uint4 cur[kStep], next[kStep], behind = make_uint4(0, 0, 0, 0);
    if (trips > 0) load(next, behind);
#pragma unroll 1
    for (int t = 0; t < trips; ++t) {
#pragma unroll
        for (int i = 0; i < kStep; ++i) cur[i] = next[i];
        const uint4 last = behind;
        if (t + 1 < trips) load(next, behind);
        if (kWords != kAligned) assemble(cur, last);
        float m = top;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const float high = largest<kBf16>(cur[i]);
            m = fmaxf(m, high);
            const uint32_t key = __reduce_max_sync(0xFFFFFFFFu, key_of(high));
            if (lane == i) mine = key;
        }
        if (lane < kStep && first_block + t * kStep + lane < p.blocks) block_max[t * kStep + lane] = from_key(mine);
        sum = __fmul_rn(sum, exp_of(top - m));  // (fused into the addition below in all forms of this code, or in none)
        top = m;
        const uint64_t minus_top = pack2(-top, -top), hi = pack2(kLog2eHi, kLog2eHi), lo = pack2(kLog2eLo, kLog2eLo);
        uint64_t sum2[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < kStep; ++i)
#pragma unroll
            for (int j = 0; j < kPer; j += 2) {
                const uint64_t d = add2(pack2(value(cur[i], j), value(cur[i], j + 1)), minus_top);
                float a, b;
                unpack2(fma2(d, lo, mul2(d, hi)), a, b);
                sum2[(j >> 1) & 1] = add2(sum2[(j >> 1) & 1], pack2(ex2_approx(a), ex2_approx(b)));
            }
        float s0, s1;
        unpack2(add2(sum2[0], sum2[1]), s0, s1);
        sum = __fadd_rn(sum, __fadd_rn(s0, s1));
    }
    const float all = from_key(__reduce_max_sync(0xFFFFFFFFu, key_of(top)));
    sum *= exp_of(top - all);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
    // a sum of 0: nothing but -inf, no candidate (the lowest value would be one)
    if (lane == 0) p.pairs[(int64_t)row * p.parts + part] = make_float2(sum == 0.f ? __uint_as_float(0xFF800000u) : all, sum);
}
// a row that begins off a 16-byte boundary
template <bool kBf16>
__device__ __noinline__ void scan_shifted(const BeamParams& p, int row, int part, int words) {
    if (kBf16 && words == 0)
        scan_segment<kBf16, 0>(p, row, part);
    else if (words == 1)
        scan_segment<kBf16, 1>(p, row, part);
    else if (words == 2)
        scan_segment<kBf16, 2>(p, row, part);
    else
        scan_segment<kBf16, 3>(p, row, part);
}

// The three levels: a group's segments, the best segments' blocks, the best blocks' logits; few blocks are
// looked at straight away, at level 0, and level 1 is left out (4 x 32000 13.3 -> 11.6 us).  A strip is what one
// row (level 0) or one of the best of the level before brings.
__device__ __forceinline__ bool few_blocks(const BeamParams& p) { return p.group * p.blocks <= kFewBlocks; }
struct Strip {
    int row, first, length;   // row -1: nothing
    const char* base;         // the item numbered `first`
    int step;                 // bytes from one to the next: 8 (pairs), 4, or 2 (bf16)
    __device__ __forceinline__ float item(int i) const {
        const char* at = base + (int64_t)i * step;
        if (step == 2) return __uint_as_float((uint32_t)__ldcg(reinterpret_cast<const unsigned short*>(at)) << 16);
        return __ldcg(reinterpret_cast<const float*>(at));
    }
};
template <bool kBf16>
__device__ __forceinline__ Strip strip_of(const BeamParams& p, const BeamShared& sh, int level, int row0, int i) {
    constexpr int kBlock = kBf16 ? 256 : 128, kSize = kBf16 ? 2 : 4;
    if (level == 0 && !few_blocks(p)) return {i, 0, p.parts, reinterpret_cast<const char*>(p.pairs + (int64_t)(row0 + i) * p.parts), 8};
    if (level == 0) return {i, 0, p.blocks, reinterpret_cast<const char*>(p.block_max + (int64_t)(row0 + i) * p.blocks), 4};
    const Found f = sh.chosen[level - (few_blocks(p) ? 2 : 1)][i];
    const int row = f.row(), at = f.index();
    if (f.score == 0 || sh.ended_row[row]) return {-1, 0, 0, nullptr, 4};
    if (level == 1) {
        const int first = at * p.trips * kStep;
        return {row, first, min(p.trips * kStep, p.blocks - first),
                reinterpret_cast<const char*>(p.block_max + (int64_t)(row0 + row) * p.blocks + first), 4};
    }
    const int64_t first = (int64_t)at * kBlock;
    return {row, (int)first, (int)(min(first + kBlock, p.vocab) - first),
            static_cast<const char*>(p.logits) + ((int64_t)(row0 + row) * p.row_stride + first) * kSize, kSize};
}

// What the list could not hold, in rounds of maximum.
template <bool kBf16>
__device__ __noinline__ void best_of_many(const BeamParams& p, BeamShared& sh, int g, int level) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row0 = g * p.group;
    const int strips = level == 0 ? p.group : p.n_out;
    Found last = {~0ull, 0};
    __syncthreads();
    for (int round = 0; round < p.n_out; ++round) {
        Found own = {0, ~0ull};
        auto offer = [&](int r, int b, float z) {
            const unsigned long long place = place_of(r, z, b);
            const Found f = {sh.score(place), place};
            if (better(last, f) && better(f, own)) own = f;
        };
        for (int i = warp; i < strips; i += kWarps) {
            const Strip t = strip_of<kBf16>(p, sh, level, row0, i);
            if (t.row < 0 || !(sh.const_of[t.row] > -INFINITY)) continue;
            for (int off = lane; off < t.length; off += 32) {
                const float z = t.item(off);
                if (z > -INFINITY) offer(t.row, t.first + off, z);
            }
        }
        for (int r = tid; r < p.group; r += kThreads)
            if (sh.ended_row[r] && sh.total_of[r] > -INFINITY) offer(r, 0, 0.f);
        for (int x = 16; x > 0; x >>= 1) {
            Found o;
            o.score = __shfl_xor_sync(0xFFFFFFFFu, own.score, x);
            o.place = __shfl_xor_sync(0xFFFFFFFFu, own.place, x);
            if (better(o, own)) own = o;
        }
        if (lane == 0) sh.warp_found[warp] = own;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w)
            if (better(sh.warp_found[w], own)) own = sh.warp_found[w];
        if (tid == 0) sh.chosen[level][round] = own;
        last = own;
        __syncthreads();
        if (own.score == 0) break;
    }
}

// the group's candidates, and what comes of them
template <bool kBf16>
__device__ __noinline__ void join_group(const BeamParams& p, int g) {
    __shared__ BeamShared sh;  // (handed in by reference it is read by generic loads, several times slower)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row0 = g * p.group;
    for (int r = warp; r < p.group; r += kWarps) {
        const float2* pairs = p.pairs + (int64_t)(row0 + r) * p.parts;
        const float2 early = __ldcg(&pairs[min(lane, p.parts - 1)]);  // (of a row without a beam: whatever stands there)
        const float t = p.totals[row0 + r];
        const bool e = p.ended != nullptr && p.ended[row0 + r] != 0;
        float top = __uint_as_float(0xFF800000u);
        double sum = 0.0;
        if (t > -INFINITY && !e) {
            for (int i = lane; i < p.parts; i += 32) {
                const float2 v = i < 32 ? early : __ldcg(&pairs[i]);
                if (v.y > 0.f) {  // (running: a row of more than 32 segments)
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
            const bool counts = top > -INFINITY && sum > 0.0;
            const double log_sum = log(sum);
            sh.ended_row[r] = e;
            sh.top_of[r] = counts ? top : 0.f;
            sh.log_of[r] = log_sum;
            sh.total_of[r] = e || counts ? (double)t : -INFINITY;
            sh.const_of[r] = counts ? (float)((double)t - log_sum) : __uint_as_float(0xFF800000u);
        }
    }
    __syncthreads();
    const float none = __uint_as_float(0xFF800000u);   // no item
#pragma unroll 1
    for (int level = 0; level < kLevels; level += few_blocks(p) ? 2 : 1) {
        const int strips = level == 0 ? p.group : p.n_out;
        Found* const chosen = sh.chosen[level];
        for (int i = tid; i < p.n_out; i += kThreads) chosen[i].score = 0;
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        float mine = none, reach = none;
        const int before = level - (few_blocks(p) ? 2 : 1);
        if (level > 0) {
            const Found f = sh.chosen[before][p.n_out - 1];
            if (f.score != 0) {
                reach = (float)from_key64(f.score);
                reach -= fabsf(reach) * 1.2e-7f;  // (rounded: a step of 2^-23)
            }
        }
        // Scores to fp32 accuracy with what they may be off by (the difference to the row's maximum, the row's
        // constant and their sum are rounded once each): a bound is taken among the least they can be,
        // and listed is what can reach it.
        auto visit = [&](bool bound) {
#pragma unroll 1
            for (int i = warp; i < strips; i += kWarps) {
                const Strip t = strip_of<kBf16>(p, sh, level, row0, i);
                if (t.row < 0) continue;
                const float c = sh.const_of[t.row], top = sh.top_of[t.row];
                if (!(c > none)) continue;
#pragma unroll 1
                for (int off = lane; off < t.length; off += 32 * kBatch) {
                    float z[kBatch];
#pragma unroll
                    for (int k = 0; k < kBatch; ++k) z[k] = t.item(min(off + k * 32, t.length - 1));
                    uint32_t hits = 0;
#pragma unroll
                    for (int k = 0; k < kBatch; ++k) {
                        const float d = z[k] - top, a = d + c, off_by = (fabsf(d) + fabsf(c)) * 2.4e-7f;  // two steps of 2^-23
                        // (d, a and a - off_by may pass the lowest number: only a logit of -inf is no candidate, and what
                        // is then not a number reaches any bound)
                        const bool real = z[k] > none && off + k * 32 < t.length;
                        if (real) mine = fmaxf(mine, fmaxf(a - off_by, kLowest));
                        hits |= (uint32_t)(real && !(a + off_by < reach)) << k;
                    }
#pragma unroll 1
                    for (hits = bound ? 0 : hits; hits != 0; hits &= hits - 1) {  // one copy of this code
                        const int k = __ffs(hits) - 1, n = atomicAdd(&sh.listed, 1);
                        float hit = z[0];
#pragma unroll
                        for (int x = 1; x < kBatch; ++x) hit = k == x ? z[x] : hit;
                        if (n < kList) sh.list[n].place = place_of(t.row, hit, t.first + off + k * 32);
                    }
                }
            }
            // ended beams: one item each
            for (int r = tid; r < p.group; r += kThreads)
                if (sh.ended_row[r] && sh.total_of[r] > -INFINITY) {
                    const float t = (float)sh.total_of[r];
                    if (bound) {
                        mine = fmaxf(mine, t);
                    } else if (!(t < reach)) {
                        const int n = atomicAdd(&sh.listed, 1);
                        if (n < kList) sh.list[n].place = place_of(r, 0.f, 0);
                    }
                }
        };
        // A few segments are ranked as they are; more want a bound first (ranking 256 takes 4 us).
        int n = 0;
#pragma unroll 1
        for (int pass = level > 0 || p.group * (few_blocks(p) ? p.blocks : p.parts) <= kRankAll ? 1 : 0; pass < 4; ++pass) {
            // 0: a bound, 1: the list; if that overflows 2: another bound, 3: the list again
            visit((pass & 1) == 0);
            if (pass == 0) {
                reach = reach_by_warps(mine, from_key(__reduce_max_sync(0xFFFFFFFFu, key_of(mine))), none, p.n_out, sh.tops,
                                       sh.bounds, sh.nths);
            } else if (pass == 2) {
                if (tid == 0) sh.listed = 0;
                reach = fmaxf(reach, reach_by_threads(mine, sh.maxima, &sh.bound, p.n_out));
            } else {
                __syncthreads();
                n = sh.listed;
                __syncthreads();
                if (n <= kList) break;
            }
        }
        if (n <= kList) {
            for (int i = tid; i < n + kRankStep; i += kThreads) {
                if (i < n) sh.list[i].score = sh.score(sh.list[i].place);
                else sh.list[i] = {0, ~0ull};  // behind the last one: not better than any
            }
            __syncthreads();
#pragma unroll 1
            for (int i = tid; i < n; i += kThreads) {
                const Found mine_now = sh.list[i];
                int rank = 0;
#pragma unroll 1
                for (int j = 0; j < n; j += kRankStep) {
                    Found x[kRankStep];
#pragma unroll
                    for (int k = 0; k < kRankStep; ++k) x[k] = sh.list[j + k];
#pragma unroll
                    for (int k = 0; k < kRankStep; ++k)
                        rank += (x[k].score > mine_now.score) | ((x[k].score == mine_now.score) & (x[k].place < mine_now.place));
                }
                if (rank < p.n_out) chosen[rank] = mine_now;
            }
            __syncthreads();
        } else {
            best_of_many<kBf16>(p, sh, g, level);
        }
    }
    if (tid < kBeamMaxGroup) sh.first_of[tid] = kBeamMaxOut;
    if (tid < 2) sh.taken[tid] = 0;
    __syncthreads();
    // ---- out: in order, or a stream's best in the stream's own place and the others in the free ones ---
    const Found f = sh.chosen[kLevels - 1][tid < p.n_out ? tid : 0];
    const bool real = tid < p.n_out && f.score != 0;
    const int r = real ? f.row() : -1;
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
        const int token = !real ? -1 : was_ended ? p.end_token : f.index();
        const int64_t at = (int64_t)g * p.n_out + place;
        p.totals_out[at] = real ? (float)from_key64(f.score) : -INFINITY;
        p.source[at] = real ? row0 + r : -1;
        p.token_ids[at] = token;
        if (p.entropy != nullptr)
            p.entropy[at] = real && !was_ended ? (float)(sh.log_of[r] - ((double)f.logit() - (double)sh.top_of[r])) : 0.f;
        if (p.ended_out != nullptr) p.ended_out[at] = real && (was_ended || (p.end_token >= 0 && token == p.end_token));
    }
}

// kAll: all rows begin at 16-byte boundaries (a kernel without the code for others: 4 x 32000 10.8 -> 10.3 us)
template <bool kBf16, bool kAll>
__global__ void __launch_bounds__(kThreads, 4) beam_kernel(const BeamParams p) {
    __shared__ int last_one;
    const int warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    // A CTA works for one group: eight of its segments, all of a row's, then the next row's.
    const int g = blockIdx.x / p.group_ctas, cta = blockIdx.x - g * p.group_ctas, segment = cta * kWarps + warp;
    const int in_group = segment / p.parts, row = g * p.group + in_group;
    if (in_group < p.group && p.totals[row] > -INFINITY && !(p.ended != nullptr && p.ended[row] != 0)) {
        const uintptr_t row_at = (uintptr_t)p.logits + (int64_t)row * p.row_stride * (kBf16 ? 2 : 4);
        const int part = segment - in_group * p.parts, words = (int)(row_at & 15) >> 2;
        if (kAll || (row_at & 15) == 0)
            scan_segment<kBf16, kAligned>(p, row, part);
        else
            scan_shifted<kBf16>(p, row, part, words);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(&p.tickets[g]) : "memory");
        last_one = before == p.group_ctas - 1;
        if (last_one) p.tickets[g] = 0;  // for the next call
    }
    __syncthreads();
    if (last_one) join_group<kBf16>(p, g);
}

}  // namespace

cudaError_t launch_beam(const BeamParams& p, cudaStream_t st) {
    TraceRange trace("sirllm:beam_select");
    cudaLaunchConfig_t cfg = {};
    BeamParams q = p;
    q.group_ctas = (p.group * p.parts + kWarps - 1) / kWarps;
    cfg.gridDim = dim3((unsigned)(p.n_streams / p.group * q.group_ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const bool bf16 = p.logits_dtype == SIRLLM_BF16;
    const bool all = (uintptr_t)p.logits % 16 == 0 && (p.n_streams == 1 || p.row_stride * (bf16 ? 2 : 4) % 16 == 0);
    if (bf16) return all ? cudaLaunchKernelEx(&cfg, beam_kernel<true, true>, q) : cudaLaunchKernelEx(&cfg, beam_kernel<true, false>, q);
    return all ? cudaLaunchKernelEx(&cfg, beam_kernel<false, true>, q) : cudaLaunchKernelEx(&cfg, beam_kernel<false, false>, q);
}

}  // namespace sirllm
