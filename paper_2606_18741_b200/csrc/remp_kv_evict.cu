// Eviction from a cache of 16-bit values by accumulated weight (rules: include/remp.h): the choice, then the move.
//
// The choice, one (sequence, KV head) to a thread block, or to a cluster of them for long sequences: weights become whole numbers of the
// same order and stay in registers, kKeys to a thread. The smallest weight that stays is found two bits at a time, from the
// top: three counts a round (packed, one reduction of a warp, one barrier; a cluster adds its blocks' counts over distributed
// shared memory). Places in the list follow from counts of (round of 32 positions, warp), so equal weights stay lowest position
// first and the list is ascending, whatever the order in which threads run.
//
// The move, in place: row i comes from position kept[i] >= i, ascending, so a chunk of rows may be written once it AND ALL BEFORE IT
// are read, and the chunks behind it are never touched by that. A thread block takes a slice of the dims of K and V of one
// (sequence, KV head) and goes through its chunks in order: the next chunk is asked for before this one is stored, and one
// barrier stands between the last load of a chunk and its first store. Slices share nothing, so they are as many as it
// takes to fill the GPU.
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

constexpr int kThreads = 1024;

// A whole number of the same order as the weight; NaN is below everything, -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    uint32_t b = __float_as_uint(x);
    if (x != x) return 0;
    if (b == 0x80000000u) b = 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sums of `x` over the thread block (1024 threads); total: of all.
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
    const int of_warp = scratch[lane];
    *total = __reduce_add_sync(0xffffffffu, of_warp);
    return __reduce_add_sync(0xffffffffu, lane < wid ? of_warp : 0) + in - x;
}

template <int kKeys, int kBlocks>
__global__ void __launch_bounds__(kThreads, 1) kv_choose_kernel(const __grid_constant__ EvictArgs a) {
    __shared__ uint32_t warp_counts[2][32][2];
    __shared__ int block_counts[2][3], totals[2], scratch[32];
    __shared__ int equal_at[kKeys * 32], stay_at[kKeys * 32];  // counts of (key of a thread, warp), then the sums before them
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

    uint32_t key[kKeys], open = 0, fixed = 0;  // positions to choose from; positions that stay anyway
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        const int at = begin + i * kThreads + tid;
        key[i] = 0;
        if (at < end) {
            if (at < first || at >= c.len - recent) fixed |= 1u << i;
            else open |= 1u << i, key[i] = order_of(weights[at]);
        }
    }

    // the smallest that stays: the largest T with `want` keys or more at or above it
    uint32_t least = 0;
    int above = 0;  // keys above it
#pragma unroll 1
    for (int bit = 30; bit >= -2; bit -= 2) {
        // the last round counts what is above T alone
        const bool last = bit < 0;
        const uint32_t t1 = last ? least + 1 : least | 1u << bit, t2 = last ? 0xffffffffu : least | 2u << bit, t3 = last ? 0xffffffffu : least | 3u << bit;
        uint32_t c12 = 0, c3 = 0;
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
            c12 += (key[i] >= t1 ? 1u : 0u) + (key[i] >= t2 ? 0x10000u : 0u);
            c3 += key[i] >= t3 ? 1u : 0u;
        }
        c12 = __reduce_add_sync(0xffffffffu, c12), c3 = __reduce_add_sync(0xffffffffu, c3);
        const int turn = bit >> 1 & 1;
        if (lane == 0) warp_counts[turn][wid][0] = c12, warp_counts[turn][wid][1] = c3;
        __syncthreads();
        c12 = warp_counts[turn][lane][0], c3 = warp_counts[turn][lane][1];
        int n1 = __reduce_add_sync(0xffffffffu, c12 & 0xffff), n2 = __reduce_add_sync(0xffffffffu, c12 >> 16), n3 = __reduce_add_sync(0xffffffffu, c3);
        if constexpr (kBlocks > 1) {
            if (tid == 0) block_counts[turn][0] = n1, block_counts[turn][1] = n2, block_counts[turn][2] = n3;
            cg::this_cluster().sync();
            n1 = n2 = n3 = 0;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const int* x = cg::this_cluster().map_shared_rank(block_counts[turn], b);
                n1 += x[0], n2 += x[1], n3 += x[2];
            }
        }
        if (last) above = least == 0xffffffffu ? 0 : n1;
        else if (n3 >= want) least = t3;
        else if (n2 >= want) least = t2;
        else if (n1 >= want) least = t1;
    }
    if (want == 0) least = 0xffffffffu, above = 0;  // nothing: no key is that large
    const int ties = want - above;

    // places: equal keys first, then all that stay
    uint32_t equal = 0;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        if ((open >> i & 1) && key[i] == least) equal |= 1u << i;
        const unsigned votes = __ballot_sync(0xffffffffu, equal >> i & 1);
        if (lane == 0) equal_at[i * 32 + wid] = __popc(votes);
    }
    const auto sum_up = [&](int* counts, int which) {  // counts of this block become sums before each, over the cluster
        __syncthreads();
        const int x = tid < kKeys * 32 ? counts[tid] : 0;
        int total, sum = sums_before(x, &total, scratch);
        if constexpr (kBlocks > 1) {
            if (tid == 0) totals[which] = total;
            cg::this_cluster().sync();
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) sum += b < part ? *cg::this_cluster().map_shared_rank(&totals[which], b) : 0;
        }
        if (tid < kKeys * 32) counts[tid] = sum;
        __syncthreads();
    };
    sum_up(equal_at, 0);
    uint32_t stays = fixed;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        const unsigned votes = __ballot_sync(0xffffffffu, equal >> i & 1);
        const int nth = equal_at[i * 32 + wid] + __popc(votes & ((1u << lane) - 1));
        if ((open >> i & 1) && (key[i] > least || ((equal >> i & 1) && nth < ties))) stays |= 1u << i;
        const unsigned all = __ballot_sync(0xffffffffu, stays >> i & 1);
        if (lane == 0) stay_at[i * 32 + wid] = __popc(all);
    }
    float weight[kKeys];  // read before anything is written
#pragma unroll
    for (int i = 0; i < kKeys; ++i) weight[i] = stays >> i & 1 ? weights[begin + i * kThreads + tid] : 0.f;
    sum_up(stay_at, 1);
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
        const unsigned all = __ballot_sync(0xffffffffu, stays >> i & 1);
        if (stays >> i & 1) {
            const int to = stay_at[i * 32 + wid] + __popc(all & ((1u << lane) - 1));
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

__global__ void __launch_bounds__(kMoveThreads, 3) kv_move_kernel(const __grid_constant__ MoveArgs m) {
    const EvictArgs& a = m.e;
    const KvView& v = a.v;
    __shared__ int64_t from_at[2][kMoveThreads * kMoveLoads / 4], to_at[2][kMoveThreads * kMoveLoads / 4];
    const int tid = threadIdx.x, unit = blockIdx.x / m.slices, slice = blockIdx.x - unit * m.slices;
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
    const auto find = [&](int i0, int turn) {  // where the rows from i0 on come from and go to
        for (int i = tid; i < rows; i += kMoveThreads) {
            int64_t from = -1, to = -1;
            if (i0 + i < c.after) {
                const int at = kept[i0 + i];
                if (at > i0 + i && at < c.len) from = place(at), to = place(i0 + i);
            }
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
    find(lo, 0);
    __syncthreads();
    load(now, 0);
    int turn = 0;
#pragma unroll 1
    for (int i0 = lo; i0 < c.after; i0 += rows, turn ^= 1) {
        find(i0 + rows, turn ^ 1);
        __syncthreads();
        load(next, turn ^ 1);
        // All loads of this chunk are done: their values are asked for before the barrier.
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) asm volatile("" ::"r"(now[i].x), "r"(now[i].y), "r"(now[i].z), "r"(now[i].w) : "memory");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) {
            const int at = i * per_load + mine;
            if (from_at[turn][at] >= 0) *reinterpret_cast<uint4*>(base + to_at[turn][at]) = now[i];
        }
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) now[i] = next[i];
        __syncthreads();  // this chunk's places are read
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
    if (units > 0x7fffffffLL / 32) return fail(REMP_ERR_SHAPE, "too many sequences and heads");
    a.v.num_seqs = tables->num_seqs, a.v.max_blocks = tables->max_blocks_per_seq;
    a.v.seq_lens = tables->seq_lens, a.v.tables = tables->block_tables, a.v.error = error;
    a.keep = keep, a.first = first, a.recent = recent, a.weights = weights, a.weights_out = weights_out, a.stride = stride;
    a.kept = kept, a.kept_stride = kept_stride, a.max_tokens = max_tokens;
    a.room = (int32_t)std::min<int64_t>((int64_t)a.v.max_blocks * pool->block_size, kKvqMost);
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (max_tokens <= 4 * kThreads) REMP_CUDA(launch_after(kv_choose_kernel<4, 1>, units, kThreads, 0, stream, a));
    else if (max_tokens <= 16 * kThreads) REMP_CUDA(launch_after(kv_choose_kernel<16, 1>, units, kThreads, 0, stream, a));
    else if (max_tokens <= 8 * 16 * kThreads) REMP_CUDA(launch_after_in_clusters(kv_choose_kernel<16, 8>, units * 8, 8, kThreads, 0, stream, a));
    else REMP_CUDA(launch_after_in_clusters(kv_choose_kernel<32, 8>, units * 8, 8, kThreads, 0, stream, a));
    // slices of 32 bytes and more, until there are four thread blocks for each SM
    m.slices = 1;
    while (m.slices < pool->head_dim / 16 && units * m.slices < 4 * sms) m.slices *= 2;
    m.pieces = 2 * (pool->head_dim / 8) / m.slices;
    REMP_CUDA(launch_after(kv_move_kernel, units * m.slices, kMoveThreads, 0, stream, m));
    return REMP_OK;
}
