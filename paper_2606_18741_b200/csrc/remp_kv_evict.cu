// Eviction from a cache of 16-bit values by accumulated weight (rules: include/remp.h): the choice, then the move.
//
// The choice, one (sequence, KV head) to a thread block, or to a cluster of them for long sequences: weights become whole numbers of the
// same order and stay in registers, kKeys to a thread. The smallest weight that stays is found by counting: the range from the
// least to the most is cut into kThreads equal stretches of a power of two, the weights in each are counted in shared memory (a cluster adds its
// blocks' counts over distributed shared memory), and the stretch that holds it is the next range: three or four rounds, eight to ten bits of
// the range each, where two bits at a time took seventeen. Places in the list follow from counts of (round of 32 positions, warp), so equal weights stay lowest
// position first and the list is ascending, whatever the order in which threads run.
//
// The move, in place: row i comes from position kept[i] >= i, ascending, so a chunk of rows may be written once it AND ALL BEFORE IT
// are read, and the chunks behind it are never touched by that. A thread block takes a slice of the dims of K and V of one
// (sequence, KV head) and goes through its chunks in order: the next chunk is asked for before this one is stored, and one
// barrier stands between the last load of a chunk and its first store. With few sequences and heads a cluster takes a slice, each of its blocks
// every 2nd to 8th chunk, and the barrier is the cluster's. Slices share nothing, so they are as many as it then takes to fill the GPU.
//
// Bound: HBM for the move (rows that move are read and written once); latency for the choice.

#include <cooperative_groups.h>

#include <algorithm>

#include "remp_kv.h"

namespace remp {

namespace {

namespace cg = cooperative_groups;

struct EvictArgs {
    KvView v;              // its batch: sequences, lengths, tables and the error word
    const int32_t* keep;
    int32_t first, recent;
    const float* weights;
    float* weights_out;
    int64_t stride;
    int32_t* kept;
    int32_t kept_stride, max_tokens, room;
};

struct Cut {  // of one sequence
    int len, after;
    bool bad;
};

__device__ __forceinline__ Cut cut_of(const EvictArgs& a, int s) {
    Cut c;
    const int len = a.v.seq_lens[s], keep = a.keep[s];
    c.after = min(len, keep);
    c.bad = len < 0 || keep < 0 || len > a.max_tokens || len > a.room || c.after > a.kept_stride;
    c.len = c.bad ? 0 : len, c.after = c.bad ? 0 : c.after;
    return c;
}

// ---- the choice ----

// A whole number of the same order as the weight; NaN is below everything, -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    uint32_t b = __float_as_uint(x);
    if (x != x) return 0;
    if (b == 0x80000000u) b = 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sums of `x` over the thread block of kWarps warps; total: of all.
template <int kWarps>
__device__ __forceinline__ int sums_before(int x, int* total, int* scratch) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    int in = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, in, d);
        if (lane >= d) in += up;
    }
    __syncthreads();  // the scratch of the last call is read
    if (lane == 31) scratch[wid] = in;
    __syncthreads();
    const int of_warp = lane < kWarps ? scratch[lane] : 0;
    *total = __reduce_add_sync(0xffffffffu, of_warp);
    return __reduce_add_sync(0xffffffffu, lane < wid ? of_warp : 0) + in - x;
}

template <int kThreads, int kKeys, int kBlocks>
__global__ void __launch_bounds__(kThreads, kKeys > 8 ? 1 : 1024 / kThreads) kv_choose_kernel(const __grid_constant__ EvictArgs a) {
    constexpr int kWarps = kThreads / 32, kCounts = kKeys * kWarps;
    static_assert(kCounts <= kThreads, "one thread to a count");
    __shared__ int counts[2][kThreads];
    __shared__ uint32_t ends[2][kWarps], block_ends[2], found[3];
    __shared__ int totals[2], scratch[kWarps];
    __shared__ int equal_at[kCounts], stay_at[kCounts];  // counts of (key of a thread, warp), then the sums before them
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int part = kBlocks > 1 ? (int)blockIdx.x % kBlocks : 0, unit = blockIdx.x / kBlocks;
    const int s = unit / a.v.kv_heads, head = unit - s * a.v.kv_heads;
    const auto meet = [] {
        if constexpr (kBlocks > 1) cg::this_cluster().sync();
        else __syncthreads();
    };
    grid_wait();
    const Cut c = cut_of(a, s);
    if (c.bad && head == 0 && part == 0 && tid == 0) kvq_error(a.v, kErrBadLength);
    const float* weights = a.weights + ((int64_t)s * a.v.kv_heads + head) * a.stride;
    float* weights_out = a.weights_out + ((int64_t)s * a.v.kv_heads + head) * a.stride;
    int32_t* kept = a.kept + ((int64_t)s * a.v.kv_heads + head) * a.kept_stride;
    for (int i = c.after + part * kThreads + tid; i < a.kept_stride; i += kBlocks * kThreads) kept[i] = -1;
    if (c.after == c.len) {  // everything stays (the whole cluster is here)
        for (int i = part * kThreads + tid; i < c.len; i += kBlocks * kThreads) {
            kept[i] = i;
            if (weights_out != weights) weights_out[i] = weights[i];
        }
        return;
    }
    const int first = min(a.first, c.after), recent = min(a.recent, c.after - first), want = c.after - first - recent;
    const int span = ((c.len + kBlocks - 1) / kBlocks + kThreads - 1) / kThreads * kThreads;  // positions of a block, at most kKeys * kThreads
    const int begin = part * span, end = min(c.len, begin + span);

    uint32_t key[kKeys], open = 0, fixed = 0, lo = 0xffffffffu, hi = 0;  // positions to choose from; positions that stay anyway
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        const int at = begin + i * kThreads + tid;
        key[i] = 0;
        if (at < end) {
            if (at < first || at >= c.len - recent) fixed |= 1u << i;
            else open |= 1u << i, key[i] = order_of(weights[at]), lo = min(lo, key[i]), hi = max(hi, key[i]);
        }
    }

    // the smallest that stays: the largest T with `want` keys or more at or above it
    uint32_t least = 0xffffffffu;  // nothing stays: no key is that large
    int above = 0;                 // keys above it
    if (want > 0) {
        lo = __reduce_min_sync(0xffffffffu, lo), hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) ends[0][wid] = lo, ends[1][wid] = hi;
        __syncthreads();
        lo = __reduce_min_sync(0xffffffffu, lane < kWarps ? ends[0][lane] : 0xffffffffu), hi = __reduce_max_sync(0xffffffffu, lane < kWarps ? ends[1][lane] : 0);
        if constexpr (kBlocks > 1) {
            if (tid == 0) block_ends[0] = lo, block_ends[1] = hi;
            cg::this_cluster().sync();
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const uint32_t* x = cg::this_cluster().map_shared_rank(block_ends, b);
                lo = min(lo, x[0]), hi = max(hi, x[1]);
            }
        }
#pragma unroll 1
        for (int turn = 0; lo < hi; turn ^= 1) {
            // stretches of 2^shift from lo on, counted from the top; the other counts are read, this block's and the cluster's
            const int shift = max(0, 32 - __clz(hi - lo) - (31 - __clz(kThreads)));
            counts[turn][tid] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kKeys; ++i)
                if ((open >> i & 1) && key[i] >= lo && key[i] <= hi) atomicAdd(&counts[turn][kThreads - 1 - ((key[i] - lo) >> shift)], 1);
            meet();
            int mine = counts[turn][tid], total;
            if constexpr (kBlocks > 1) {
                mine = 0;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) mine += cg::this_cluster().map_shared_rank(counts[turn], b)[tid];
            }
            const int before = above + sums_before<kWarps>(mine, &total, scratch);
            if (before < want && before + mine >= want) found[0] = kThreads - 1 - tid, found[1] = before;
            __syncthreads();
            above = found[1];
            lo += found[0] << shift;
            hi = lo + min(hi - lo, (1u << shift) - 1);
        }
        least = lo;
    }
    const int ties = want - above;

    // places: equal keys first, then all that stay
    uint32_t equal = 0;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        if ((open >> i & 1) && key[i] == least) equal |= 1u << i;
        const unsigned votes = __ballot_sync(0xffffffffu, equal >> i & 1);
        if (lane == 0) equal_at[i * kWarps + wid] = __popc(votes);
    }
    const auto sum_up = [&](int* counts, int which) {  // counts of this block become sums before each, over the cluster
        __syncthreads();
        const int x = tid < kCounts ? counts[tid] : 0;
        int total, sum = sums_before<kWarps>(x, &total, scratch);
        if constexpr (kBlocks > 1) {
            if (tid == 0) totals[which] = total;
            cg::this_cluster().sync();
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) sum += b < part ? *cg::this_cluster().map_shared_rank(&totals[which], b) : 0;
        }
        if (tid < kCounts) counts[tid] = sum;
        __syncthreads();
    };
    sum_up(equal_at, 0);
    uint32_t stays = fixed;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        const unsigned votes = __ballot_sync(0xffffffffu, equal >> i & 1);
        const int nth = equal_at[i * kWarps + wid] + __popc(votes & ((1u << lane) - 1));
        if ((open >> i & 1) && (key[i] > least || ((equal >> i & 1) && nth < ties))) stays |= 1u << i;
        const unsigned all = __ballot_sync(0xffffffffu, stays >> i & 1);
        if (lane == 0) stay_at[i * kWarps + wid] = __popc(all);
    }
    float weight[kKeys];  // read before anything is written
#pragma unroll
    for (int i = 0; i < kKeys; ++i) weight[i] = stays >> i & 1 ? weights[begin + i * kThreads + tid] : 0.f;
    sum_up(stay_at, 1);
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        const unsigned all = __ballot_sync(0xffffffffu, stays >> i & 1);
        if (stays >> i & 1) {
            const int to = stay_at[i * kWarps + wid] + __popc(all & ((1u << lane) - 1));
            kept[to] = begin + i * kThreads + tid, weights_out[to] = weight[i];
        }
    }
    meet();  // nobody leaves while its counts are read
}

// ---- the move ----

constexpr int kMoveThreads = 256, kMoveLoads = 8;

struct MoveArgs {
    EvictArgs e;
    int32_t slices, pieces;  // parts of the dims, 16-byte pieces of K and V of a row in one of them (a power of two)
};

template <int kBlocks>
__global__ void __launch_bounds__(kMoveThreads, 2) kv_move_kernel(const __grid_constant__ MoveArgs m) {
    const EvictArgs& a = m.e;
    const KvView& v = a.v;
    constexpr int kMostRows = kMoveThreads * kMoveLoads / 4, kTurns = 4, kMine = kMostRows / kMoveThreads;
    __shared__ int64_t from_at[kTurns][kMostRows], to_at[kTurns][kMostRows];
    const int tid = threadIdx.x, part = (int)blockIdx.x % kBlocks, unit = blockIdx.x / kBlocks / m.slices, slice = blockIdx.x / kBlocks - unit * m.slices;
    const int s = unit / v.kv_heads, head = unit - s * v.kv_heads;
    grid_wait();
    const Cut c = cut_of(a, s);
    if (c.after == c.len) return;
    const int32_t* kept = a.kept + ((int64_t)s * v.kv_heads + head) * a.kept_stride;
    const int32_t* row = v.tables + (int64_t)s * v.max_blocks;
    const int per_load = kMoveThreads / m.pieces, rows = per_load * kMoveLoads;  // rows of one load, of a chunk
    const int half = m.pieces / 2, piece = tid % m.pieces, mine = tid / m.pieces;
    uint8_t* const base = v.base + (int64_t)head * v.s_head + (piece >= half ? v.s_kv : 0) + (slice * half + piece % half) * 16;
    const auto place = [&](int at) -> int64_t {  // of a position, or -1: its block is not in the pool
        const int tile = at / kKvqTile, in_row = tile / v.block_tiles, id = row[in_row];
        if ((uint32_t)id >= (uint32_t)v.nb) {
            kvq_error(v, kErrBadBlock);
            return -1;
        }
        return (int64_t)id * v.s_block + (int64_t)(at - in_row * v.block_tiles * kKvqTile) * v.s_token;
    };
    const auto ask = [&](int i0, int (&at)[kMine]) {  // positions that this thread's rows of the chunk from i0 on come from
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int i = tid + x * kMoveThreads;
            at[x] = i < rows && i0 + i < c.after ? kept[i0 + i] : -1;
        }
    };
    const auto find = [&](int i0, const int (&at)[kMine], int turn) {  // where these rows come from and go to
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int i = tid + x * kMoveThreads;
            if (i >= rows) continue;
            int64_t from = -1, to = -1;
            if (at[x] > i0 + i && at[x] < c.len) from = place(at[x]), to = place(i0 + i);
            from_at[turn][i] = to < 0 ? -1 : from, to_at[turn][i] = to;
        }
    };
    const auto load = [&](uint4 (&x)[kMoveLoads], int turn) {
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) {
            const int64_t from = from_at[turn][i * per_load + mine];
            x[i] = from >= 0 ? __ldcs(reinterpret_cast<const uint4*>(base + from)) : make_uint4(0, 0, 0, 0);
        }
    };
    // rows in front that stay where they are: kept[i] - i only grows
    int lo = 0, hi = c.after;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (kept[mid] == mid) lo = mid + 1;
        else hi = mid;
    }
    if (lo == c.after) return;
    uint4 now[kMoveLoads], next[kMoveLoads];
    int at[kMine];
    const int step = kBlocks * rows;
    lo += part * rows;  // this block's first chunk
    ask(lo, at);
    find(lo, at, 0);
    ask(lo + step, at);
    find(lo + step, at, 1);
    ask(lo + 2 * step, at);
    __syncthreads();
    load(now, 0);
    int turn = 0;
#pragma unroll 1
    for (int i0 = lo; i0 - part * rows < c.after; i0 += step, turn = (turn + 1) % kTurns) {
        // the next chunk's loads, the places of the one behind it, the positions of the one behind that
        load(next, (turn + 1) % kTurns);
        find(i0 + 2 * step, at, (turn + 2) % kTurns);
        ask(i0 + 3 * step, at);
        // All loads of this chunk are done: their values are asked for before the barrier. Those of the next may be on their way: they
        // come from behind what this chunk overwrites. The places that the others may still store by are three turns back.
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) asm volatile("" ::"r"(now[i].x), "r"(now[i].y), "r"(now[i].z), "r"(now[i].w) : "memory");
        if constexpr (kBlocks > 1) cg::this_cluster().sync();
        else __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) {
            const int r = i * per_load + mine;
            if (from_at[turn][r] >= 0) *reinterpret_cast<uint4*>(base + to_at[turn][r]) = now[i];
        }
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) now[i] = next[i];
    }
}

}  // namespace

}  // namespace remp

using namespace remp;

extern "C" remp_status remp_kv_evict(const remp_kv_pool* pool, const remp_block_tables* tables, const int32_t* keep, int32_t first,
                                     int32_t recent, const float* weights, float* weights_out, int64_t stride, int32_t* kept,
                                     int32_t kept_stride, int32_t max_tokens, uint32_t* error, void* stream_) {
    MoveArgs m{};
    EvictArgs& a = m.e;
    if (!tables) return fail(REMP_ERR_INVALID_ARG, "null tables");
    if (remp_status st = kv_pool_view(pool, &a.v)) return st;
    if (tables->num_seqs < 0 || tables->max_blocks_per_seq < 0) return fail(REMP_ERR_INVALID_ARG, "negative table dimensions");
    if (first < 0 || recent < 0) return fail(REMP_ERR_INVALID_ARG, "negative number of first or recent tokens");
    if (stride < 0 || kept_stride < 0 || max_tokens < 0) return fail(REMP_ERR_INVALID_ARG, "negative stride or max_tokens");
    if (max_tokens > stride || max_tokens > 1 << 18) return fail(REMP_ERR_SHAPE, "max_tokens must be at most 2^18 and at most stride");
    if (tables->num_seqs == 0) return REMP_OK;
    if (!tables->seq_lens || (tables->max_blocks_per_seq > 0 && !tables->block_tables) || !keep)
        return fail(REMP_ERR_INVALID_ARG, "null seq_lens, block_tables or keep");
    if ((max_tokens > 0 && (!weights || !weights_out)) || (kept_stride > 0 && !kept)) return fail(REMP_ERR_INVALID_ARG, "null weights or kept");
    const int64_t units = (int64_t)tables->num_seqs * pool->kv_heads;
    if (units > 0x7fffffffLL / 128) return fail(REMP_ERR_SHAPE, "too many sequences and heads");
    a.v.num_seqs = tables->num_seqs, a.v.max_blocks = tables->max_blocks_per_seq;
    a.v.seq_lens = tables->seq_lens, a.v.tables = tables->block_tables, a.v.error = error;
    a.keep = keep, a.first = first, a.recent = recent, a.weights = weights, a.weights_out = weights_out, a.stride = stride;
    a.kept = kept, a.kept_stride = kept_stride, a.max_tokens = max_tokens;
    a.room = (int32_t)std::min<int64_t>((int64_t)a.v.max_blocks * pool->block_size, kKvqMost);
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    // a thread has 4 to 16 weights, 32 where a cluster of 1024 threads each needs it
    if (max_tokens <= 1024) REMP_CUDA(launch_after(kv_choose_kernel<256, 4, 1>, units, 256, 0, stream, a));
    else if (max_tokens <= 4096) REMP_CUDA(launch_after(kv_choose_kernel<512, 8, 1>, units, 512, 0, stream, a));
    else if (max_tokens <= 16384) REMP_CUDA(launch_after(kv_choose_kernel<1024, 16, 1>, units, 1024, 0, stream, a));
    else if (max_tokens <= 32768) REMP_CUDA(launch_after_in_clusters(kv_choose_kernel<512, 8, 8>, units * 8, 8, 512, 0, stream, a));
    else if (max_tokens <= 131072) REMP_CUDA(launch_after_in_clusters(kv_choose_kernel<1024, 16, 8>, units * 8, 8, 1024, 0, stream, a));
    else REMP_CUDA(launch_after_in_clusters(kv_choose_kernel<1024, 32, 8>, units * 8, 8, 1024, 0, stream, a));
    // clusters of up to 8 thread blocks, then slices of 32 bytes and more, until there are two thread blocks for each SM
    int blocks = 1;
    while (blocks < 8 && units * blocks < 2 * sms) blocks *= 2;
    m.slices = 1;
    while (m.slices < pool->head_dim / 16 && units * blocks * m.slices < 2 * sms) m.slices *= 2;
    m.pieces = 2 * (pool->head_dim / 8) / m.slices;
    const auto move = blocks == 1 ? kv_move_kernel<1> : blocks == 2 ? kv_move_kernel<2> : blocks == 4 ? kv_move_kernel<4> : kv_move_kernel<8>;
    REMP_CUDA(launch_after_in_clusters(move, units * blocks * m.slices, blocks, kMoveThreads, 0, stream, m));
    return REMP_OK;
}
