// Streams that go on from other streams of their group, in place: stream d takes over the slots
// [shared, live_len[source[d]]) of stream source[d] in every plane of K and V, the scores and tags of
// those slots, and the length.
//
// Bytes are all there is: a source's rows are read once, whatever the number of streams that take
// them over, and written once per stream.  Rows of a plane are contiguous, so a unit of work is one
// piece of a plane's rows of one source: one bulk copy (TMA) into shared memory, one out of it per
// taker, no thread touches the data.  Where streams of a group exchange their contents (a stream that
// is overwritten is a source too), a unit is the same, shorter piece of ALL sources of the group, and
// nothing of it is written before all of it has arrived: no copy of the cache is needed, and units
// never depend on one another.
// A warp is a CTA with a ring of its own (6 pieces of 8 KB, four such CTAs to an SM).
// Measured: two of four streams forked in each of four groups, 600 slots x 512 planes of 256 bytes, 1.25 GB in 182 us
// (1.05 of the copy rate, sources in L2); one stream to seven others, 1.07 GB in 189 us (0.86: seven of eight bytes are
// written); 30 slots x 64 planes of 128 bytes 5.9 us.  Exchanges, 600 slots x 512 planes: 4 x 8 streams 5.7 TB/s (0.87); one group of
// 64 streams 1.9 TB/s (0.29: its pieces are 128 bytes).
#include "common.cuh"

namespace sirllm {

namespace {

constexpr int kPiece = 8192;
constexpr int kRing = 6, kLead = 4;  // pieces of the ring; how far loads run ahead of stores
constexpr int kSide = 2048;          // room for scores and tags on their way
constexpr int kMaxGroup = SIRLLM_MAX_GROUP;
constexpr int kCtasPerSm = 4;

__global__ void __launch_bounds__(32) reorder_kernel(const ReorderParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t full[kRing];
    __shared__ int len_of[kMaxGroup];             // length a stream takes over, -1: it stays
    __shared__ short src_of[kMaxGroup];           // taker: index of its source among the sources
    __shared__ short src_stream[kMaxGroup], index_of[kMaxGroup];
    __shared__ int src_len[kMaxGroup];            // slots to copy end here
    __shared__ unsigned char is_source[kMaxGroup];
    const int lane = threadIdx.x;
    unsigned char* const side = smem + kRing * kPiece;
    if (lane == 0) {
        for (int i = 0; i < kRing; ++i) mbar_init(&full[i], 1);
        mbar_init_fence();
    }
    grid_dependency_wait();
    const int g = blockIdx.x / p.ctas, c = blockIdx.x - g * p.ctas;
    const int row0 = g * p.group;
    // ---- what the group has to move -----------------------------------------------------------
    const int lo = p.shared_len != nullptr ? p.shared_len[g] : 0;
    const bool lo_ok = lo >= 0 && lo <= p.capacity;
    int problems = lo_ok ? 0 : SIRLLM_STATUS_OVERFLOW;
    for (int j = lane; j < p.group; j += 32) is_source[j] = 0;
    __syncwarp();
    for (int j = lane; j < p.group; j += 32) {
        const int s = p.source[row0 + j];
        int len = -1;
        if (s != -1 && s != row0 + j && lo_ok) {
            if (s < row0 || s >= row0 + p.group) {
                problems |= SIRLLM_STATUS_BAD_SOURCE;
            } else {
                len = p.live_len[s];
                if (len < 0 || len > p.capacity) {
                    problems |= SIRLLM_STATUS_OVERFLOW;
                    len = -1;
                } else if (len > lo) {
                    is_source[s - row0] = 1;
                }
            }
        }
        len_of[j] = len;
        src_of[j] = (short)(len > lo ? s - row0 : -1);
    }
    if (c == 0) {
        problems = __reduce_or_sync(0xFFFFFFFFu, problems);
        if (lane == 0 && problems) atomicOr(p.status, problems);
    }
    __syncwarp();
    int n_src = 0, end_all = 0;
    bool exchange = false;
    for (int j0 = 0; j0 < p.group; j0 += 32) {
        const int j = j0 + lane;
        const bool on = j < p.group && is_source[j];
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, on);
        if (on) {
            const int i = n_src + __popc(vote & ((1u << lane) - 1u));
            const int len = p.live_len[row0 + j];
            src_stream[i] = (short)j;
            src_len[i] = len;
            index_of[j] = (short)i;
            end_all = max(end_all, len);
            exchange |= src_of[j] >= 0;
        }
        n_src += __popc(vote);
    }
    end_all = __reduce_max_sync(0xFFFFFFFFu, end_all);
    exchange = __any_sync(0xFFFFFFFFu, exchange);
    __syncwarp();
    for (int j = lane; j < p.group; j += 32)
        if (src_of[j] >= 0) src_of[j] = index_of[src_of[j]];
    __syncwarp();

    bool ok = true;
    if (n_src > 0) {
        // ---- K and V: units numbered piece fastest, then source, then plane ---------------------
        const int width = exchange ? n_src : 1, subs = exchange ? 1 : n_src;
        const int64_t first = (int64_t)lo * p.row_bytes, range = (int64_t)end_all * p.row_bytes - first;
        const int piece = exchange ? kPiece / n_src / 16 * 16 : kPiece;
        const int pieces = (int)((range + piece - 1) / piece);
        const int tensors = (p.k != nullptr) + (p.v != nullptr), planes = tensors * p.planes;
        struct At {
            int piece, sub, plane;
        };
        auto split = [&](int n) {
            const int rest = n / pieces;
            return At{n - rest * pieces, rest % subs, rest / subs};
        };
        const At step = split(p.ctas);
        auto advance = [&](At& a) {
            a.piece += step.piece;
            a.sub += step.sub;
            a.plane += step.plane;
            if (a.piece >= pieces) {
                a.piece -= pieces;
                ++a.sub;
            }
            if (a.sub >= subs) {
                a.sub -= subs;
                ++a.plane;
            }
        };
        auto bytes_of = [&](const At& a, int i) {  // of source i in this unit
            const int64_t left = (int64_t)src_len[i] * p.row_bytes - (first + (int64_t)a.piece * piece);
            return left <= 0 ? 0 : left < piece ? (int)left : piece;
        };
        auto address = [&](const At& a, int stream) {
            char* base = a.plane < p.planes && p.k != nullptr ? p.k : p.v;
            const int plane = a.plane < p.planes ? a.plane : a.plane - p.planes;
            return base + ((int64_t)(row0 + stream) * p.planes + plane) * p.capacity * p.row_bytes + first +
                   (int64_t)a.piece * piece;
        };
        At ahead = split(c);
        int loaded = 0;
        auto load = [&]() {
            if (ahead.plane >= planes) return;
            const int stage = loaded % kRing;
            const int i0 = width == 1 ? ahead.sub : 0;
            int bytes = 0;
            for (int i = lane; i < width; i += 32) bytes += bytes_of(ahead, i0 + i);
            bytes = __reduce_add_sync(0xFFFFFFFFu, bytes);
            if (lane == 0) mbar_expect_tx(&full[stage], bytes);
            __syncwarp();
            for (int i = lane; i < width; i += 32) {
                const int n = bytes_of(ahead, i0 + i);
                if (n > 0)
                    bulk_load(smem + stage * kPiece + i * piece, address(ahead, src_stream[i0 + i]), n, &full[stage]);
            }
            ++loaded;
            advance(ahead);
        };
        for (int i = 0; i < kLead; ++i) load();
        At at = split(c);
        int done = 0;
        for (; at.plane < planes; advance(at), ++done) {
            const int stage = done % kRing;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&full[stage], (done / kRing) & 1, kMbarSpinLimit));
            if (!ok) break;
            for (int j = lane; j < p.group; j += 32) {
                const int i = src_of[j];
                if (i < 0 || (width == 1 && i != at.sub)) continue;
                const int n = bytes_of(at, i);
                if (n > 0) bulk_store(address(at, j), smem + stage * kPiece + (width == 1 ? 0 : i) * piece, n);
            }
            bulk_commit();
            // the next load goes where the stores of kRing - kLead units ago came from
            bulk_wait_read<kRing - kLead>();
            __syncwarp();
            load();
        }
        if (!ok) {
            if (lane == 0) atomicOr(p.status, SIRLLM_STATUS_TIMEOUT);
            for (int i = done; i < loaded; ++i)  // let the copies in flight land
                mbar_wait_bounded(&full[i % kRing], (i / kRing) & 1, 1u << 14);
        }
        // ---- scores and tags: a lane has one slot of all streams of the group --------------------
        const int lanes = min(32, kSide / (8 * n_src));
        for (int t = 0; t < 2 && ok; ++t) {
            if (t == 0 ? p.scores == nullptr : p.serial == nullptr) continue;
            unsigned long long* mine = reinterpret_cast<unsigned long long*>(side) + lane;
            for (int64_t slot = lo + (int64_t)c * lanes + lane; lane < lanes && slot < end_all;
                 slot += (int64_t)p.ctas * lanes) {
#pragma unroll 4
                for (int i = 0; i < n_src; ++i) {
                    const int64_t from = (int64_t)(row0 + src_stream[i]) * p.capacity + slot;
                    if (slot < src_len[i])
                        mine[i * lanes] = t == 0 ? (unsigned long long)__float_as_uint(p.scores[from])
                                                 : (unsigned long long)p.serial[from];
                }
                for (int j = 0; j < p.group; ++j) {
                    const int i = src_of[j];
                    if (i < 0 || slot >= src_len[i]) continue;
                    const int64_t to = (int64_t)(row0 + j) * p.capacity + slot;
                    if (t == 0)
                        p.scores[to] = __uint_as_float((uint32_t)mine[i * lanes]);
                    else
                        p.serial[to] = (int64_t)mine[i * lanes];
                }
            }
            __syncwarp();
        }
        bulk_wait_all();
    }
    // ---- lengths: once every CTA of the group has read them ---------------------------------------
    __syncwarp();
    int last = 0;
    if (lane == 0) {
        int before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(&p.tickets[g]) : "memory");
        last = before == p.ctas - 1;
        if (last) p.tickets[g] = 0;  // for the next call
    }
    if (!__shfl_sync(0xFFFFFFFFu, last, 0)) return;
    for (int j = lane; j < p.group; j += 32)
        if (len_of[j] >= 0) p.live_len[row0 + j] = len_of[j];
}

}  // namespace

cudaError_t launch_reorder(const ReorderParams& p, cudaStream_t st) {
    TraceRange trace("sirllm:reorder_streams");
    static unsigned char allowed[kMaxDevices];
    DeviceProps dp;
    cudaError_t e = device_props(&dp);
    if (e != cudaSuccess) return e;
    e = allow_max_dynamic_smem((const void*)reorder_kernel, dp, allowed);
    if (e != cudaSuccess) return e;
    ReorderParams q = p;
    const int groups = p.n_streams / p.group;
    // Two waves of CTAs: a group without moves leaves its room to others, and SMs differ in speed.  But no more
    // than have eight pieces each if all streams move whole planes: 1184 CTAs of which a hundred had work
    // took 2 us for their arrivals alone.
    const int64_t pieces = ((int64_t)p.capacity * p.row_bytes + kPiece - 1) / kPiece * p.planes *
                           ((p.k != nullptr) + (p.v != nullptr)) * p.group;
    const int64_t waves = (2 * kCtasPerSm * dp.n_sm + groups - 1) / groups;
    q.ctas = (int)(pieces / 8 + 1 < waves ? pieces / 8 + 1 : waves);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * q.ctas));
    cfg.blockDim = dim3(32);
    cfg.dynamicSmemBytes = kRing * kPiece + kSide;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, reorder_kernel, q);
}

}  // namespace sirllm
