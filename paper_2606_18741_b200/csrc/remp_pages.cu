// Pages of a cache between two switches: fork, free, compact (tables and reference counts) and the copy of the pages
// that these name (include/remp.h). Everything stays on the device: counts are read by the next kernel, not by the host.
//
// Numbering: a free id's place among the free ids is id - (blocks in use below it), so fork's "lowest free ids first" and
// compact's "blocks above N, in order, to free ids below N, in order" are prefix sums over the reference counts. They
// are taken in chunks of 1024 blocks: counts of all chunks, then every thread block adds up the counts before its chunk by
// itself. No block waits for another, and the result is the same in any order.
//
// Bound: latency of the launches (tables and counts are a few MB at most), so small inputs take ONE launch of one thread
// block that walks the chunks, large ones a launch for each step. Measured: fork of 8 children 7.4 us (profiled);
// free and compaction of 4096 blocks and 128 sequences of 32 blocks 3.3 and 6.7 us each in a graph. The copy is bound by HBM: 1.05 GB in 166 us, 6.3 TB/s.

#include <algorithm>

#include "remp_launch.h"

namespace remp {

namespace {

constexpr int kChunk = 1024;  // blocks of a chunk = threads of a thread block

// One launch up to here (entries: rows to write x table width). Above, the steps spread over the GPU. A call from an idle
// GPU, one launch / spread, us (free, compact, fork): 600 blocks and 32 x 16 entries 13.3 / 15.4, 13.7 / 20.9, 14.5 / 21.4;
// 2048 and 64 x 32 13.6 / 15.3, 17.5 / 21.0, 15.9 / 21.2; 4096 and 128 x 32 17.4 / 15.2, 23.9 / 21.0, 18.2 / 21.3; 8192 and
// 256 x 32 23.7 / 15.3, 32.1 / 21.0, 24.1 / 21.3. In a graph spread wins from 2048 blocks (compact 6.9 / 6.6, at 8192 22.1 / 6.9).
constexpr int64_t kSoloBlocks = 2048, kSoloEntries = 2048, kSoloForks = 1024;

// Exclusive count of `flag` over the thread block (kChunk threads).
__device__ __forceinline__ int rank_in_block(bool flag) {
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const unsigned votes = __ballot_sync(0xffffffffu, flag);
    __syncthreads();  // sums of the last call are read
    if (lane == 0) sums[wid] = __popc(votes);
    __syncthreads();
    int mine = lane < wid ? sums[lane] : 0;
    mine = __reduce_add_sync(0xffffffffu, mine);
    return mine + __popc(votes & ((1u << lane) - 1));
}

// Sum of x over the thread block.
__device__ __forceinline__ int sum_of_block(int x) {
    __shared__ int sums[32];
    x = __reduce_add_sync(0xffffffffu, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = x;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, sums[threadIdx.x & 31]);
}

__device__ __forceinline__ int sum_of_counts(const int* counts, int n) {
    int x = 0;
    for (int i = threadIdx.x; i < n; i += kChunk) x += counts[i];
    return sum_of_block(x);
}

// Blocks that a sequence of `len` tokens has; -1: a length that its row does not hold.
__device__ __forceinline__ int need_of(int len, int block_size, int max_blocks) {
    if (len < 0) return -1;
    const int need = len / block_size + (len % block_size != 0);
    return need <= max_blocks ? need : -1;
}

// ---------------------------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------------------------

struct Fork {
    int32_t *lens, *tables;
    int32_t num_seqs, width, block_size;
    const int32_t *parents, *children;
    int32_t m;
    const int32_t* refs;
    int32_t* refs_out;
    int32_t nb;
    int2* pairs;
    int32_t* result;
    // scratch
    int *counts, *nth, *ids, *words;  // free blocks of a chunk; child's place among those that need one; ids; need, bad
};

__device__ __forceinline__ void fork_count(const Fork& f, int chunk) {
    const int id = chunk * kChunk + threadIdx.x;
    const int r = id < f.nb ? f.refs[id] : 1;
    if (id < f.nb && f.refs_out != f.refs) f.refs_out[id] = r;
    const int n = __syncthreads_count(r == 0);
    if (threadIdx.x == 0) f.counts[chunk] = n;
}

// Which children need a block of their own, and the place of each among them.
__device__ __forceinline__ void fork_children(const Fork& f) {
    int carry = 0, bad = 0;
    for (int base = 0; base < f.m; base += kChunk) {
        const int i = base + threadIdx.x;
        bool part = false;
        if (i < f.m) {
            const int p = f.parents[i], c = f.children[i];
            const int len = p >= 0 && p < f.num_seqs ? f.lens[p] : -1;
            if (c < 0 || c >= f.num_seqs || need_of(len, f.block_size, f.width) < 0) bad = 1;
            part = len > 0 && len % f.block_size != 0;
            f.pairs[i] = make_int2(-1, -1);
        }
        const int r = rank_in_block(part);
        if (i < f.m) f.nth[i] = part ? carry + r : -1;
        carry += __syncthreads_count(part);
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) f.words[0] = carry, f.words[1] = bad;
}

__device__ __forceinline__ void fork_ids(const Fork& f, int chunk, int chunks) {
    const int before = sum_of_counts(f.counts, chunk);
    const int id = chunk * kChunk + threadIdx.x;
    const bool is_free = id < f.nb && f.refs[id] == 0;
    const int r = before + rank_in_block(is_free);
    if (is_free && r < f.m) f.ids[r] = id;
    if (chunk == chunks - 1 && threadIdx.x == 0) {
        const int need = f.words[0], bad = f.words[1];
        const bool room = need <= before + f.counts[chunk];
        f.words[2] = !bad && room;
        f.result[0] = !bad && room ? need : 0;
        f.result[1] = (bad ? kErrBadLength : 0) | (room ? 0 : kErrCapacity);
    }
}

__device__ __forceinline__ void fork_row(const Fork& f, int i, int lane) {
    if (!f.words[2]) return;
    const int p = f.parents[i], c = f.children[i], len = f.lens[p];
    const int need = need_of(len, f.block_size, f.width), nth = f.nth[i];
    const int32_t* from = f.tables + (int64_t)p * f.width;
    int32_t* to = f.tables + (int64_t)c * f.width;
    for (int j = lane; j < f.width; j += 32) {
        int b = -1;
        if (j < need) {
            b = from[j];
            if (j == need - 1 && nth >= 0) {
                const int fresh = f.ids[nth];
                f.pairs[nth] = make_int2(b, fresh);
                if (b < 0 || b >= f.nb) atomicOr(reinterpret_cast<uint32_t*>(f.result + 1), (uint32_t)kErrBadBlock);
                b = fresh;
            }
            if (b >= 0 && b < f.nb) atomicAdd(f.refs_out + b, 1);
            else atomicOr(reinterpret_cast<uint32_t*>(f.result + 1), (uint32_t)kErrBadBlock);
        }
        to[j] = b;
    }
    if (lane == 0) f.lens[c] = len;
}

__global__ void __launch_bounds__(kChunk) fork_solo_kernel(Fork f, int chunks) {
    __shared__ int counts[kSoloBlocks / kChunk], nth[kSoloForks], ids[kSoloForks], words[3];
    f.counts = counts, f.nth = nth, f.ids = ids, f.words = words;
    grid_wait();
    for (int c = 0; c < chunks; ++c) fork_count(f, c);
    fork_children(f);
    __syncthreads();
    for (int c = 0; c < chunks; ++c) fork_ids(f, c, chunks);
    __syncthreads();
    for (int i = threadIdx.x >> 5; i < f.m; i += kChunk / 32) fork_row(f, i, threadIdx.x & 31);
}

__global__ void __launch_bounds__(kChunk) fork_count_kernel(Fork f, int chunks) {
    grid_wait();
    if ((int)blockIdx.x < chunks) fork_count(f, blockIdx.x);
    else fork_children(f);
}
__global__ void __launch_bounds__(kChunk) fork_ids_kernel(Fork f, int chunks) {
    grid_wait();
    fork_ids(f, blockIdx.x, chunks);
}
__global__ void __launch_bounds__(256) fork_rows_kernel(Fork f) {
    grid_wait();
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (i < f.m) fork_row(f, i, threadIdx.x & 31);
}

// ---------------------------------------------------------------------------------------------
// free
// ---------------------------------------------------------------------------------------------

struct Free {
    const int32_t *lens, *tables;
    int32_t num_seqs, width, block_size;
    const int32_t *finished, *refs;
    int32_t nb;
    int32_t *lens_out, *tables_out, *refs_out, *result;
};

__device__ __forceinline__ void free_begin(const Free& f, int64_t at, int64_t step) {
    if (f.refs_out != f.refs)
        for (int64_t i = at; i < f.nb; i += step) f.refs_out[i] = f.refs[i];
    if (at == 0) f.result[0] = f.result[1] = 0;
}

// One warp, one sequence: every entry is read and written by the same lane, so outputs may be inputs.
__device__ __forceinline__ void free_row(const Free& f, int s, int lane) {
    const int len = f.lens[s], need = need_of(len, f.block_size, f.width);
    const bool done = f.finished[s] != 0;
    const int64_t row = (int64_t)s * f.width;
    uint32_t bad = done && need < 0 ? (uint32_t)kErrBadLength : 0;
    int freed = 0;
    for (int j = lane; j < f.width; j += 32) {
        int b = f.tables[row + j];
        if (done) {
            if (j < need) {
                if (b < 0 || b >= f.nb) {
                    bad |= kErrBadBlock;
                } else {
                    const int was = atomicSub(f.refs_out + b, 1);
                    freed += was == 1;
                    if (was <= 0) bad |= kErrBadBlock;
                }
            }
            b = -1;
        }
        f.tables_out[row + j] = b;
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    freed = __reduce_add_sync(0xffffffffu, freed);
    if (lane == 0) {
        f.lens_out[s] = done ? 0 : len;
        if (freed) atomicAdd(f.result, freed);
        if (bad) atomicOr(reinterpret_cast<uint32_t*>(f.result + 1), bad);
    }
}

__global__ void __launch_bounds__(kChunk) free_solo_kernel(Free f) {
    grid_wait();
    free_begin(f, threadIdx.x, kChunk);
    __syncthreads();
    for (int s = threadIdx.x >> 5; s < f.num_seqs; s += kChunk / 32) free_row(f, s, threadIdx.x & 31);
}
__global__ void __launch_bounds__(256) free_begin_kernel(Free f) {
    grid_wait();
    free_begin(f, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
__global__ void __launch_bounds__(256) free_rows_kernel(Free f) {
    grid_wait();
    const int s = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (s < f.num_seqs) free_row(f, s, threadIdx.x & 31);
}

// ---------------------------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------------------------

struct Compact {
    const int32_t *lens, *tables;
    int32_t num_seqs, width, block_size;
    const int32_t* refs;
    int32_t nb;
    int32_t *tables_out, *refs_out;
    int2* pairs;
    int32_t max_pairs;
    int32_t* result;
    // scratch: blocks in use of a chunk; the counts as they were (refs_out may be refs); a moved block's, or a filled
    // id's, place in `pairs`
    int *counts, *was, *place;
};

__device__ __forceinline__ void compact_count(const Compact& c, int chunk) {
    const int id = chunk * kChunk + threadIdx.x;
    const int r = id < c.nb ? c.refs[id] : 0;
    if (id < c.nb) c.was[id] = r;
    const int n = __syncthreads_count(r > 0);
    if (threadIdx.x == 0) c.counts[chunk] = n;
}

__device__ __forceinline__ void compact_assign(const Compact& c, int chunk, int chunks) {
    const int total = sum_of_counts(c.counts, chunks), before = sum_of_counts(c.counts, chunk);
    const int last = total / kChunk;  // the chunk that id `total` is in
    int below = sum_of_counts(c.counts, min(last, chunks));
    const int edge = last * kChunk + threadIdx.x;
    below += __syncthreads_count(edge < total && edge < c.nb && c.was[edge] > 0);  // blocks in use below `total`
    const int id = chunk * kChunk + threadIdx.x;
    const bool used = id < c.nb && c.was[id] > 0;
    const int r = before + rank_in_block(used);
    if (id < c.nb) {
        if (used && id >= total) {
            c.place[id] = r - below;
            c.pairs[r - below].x = id;
        } else if (!used && id < total) {
            c.place[id] = id - r;
            c.pairs[id - r].y = id;
        }
        // every chunk clears its share of what is behind the list
        if (id < c.max_pairs && id >= total - below) c.pairs[id] = make_int2(-1, -1);
    }
    for (int i = c.nb + threadIdx.x; chunk == chunks - 1 && i < c.max_pairs; i += kChunk) c.pairs[i] = make_int2(-1, -1);
    if (chunk == 0 && threadIdx.x == 0) c.result[0] = total - below, c.result[1] = 0;
}

__device__ __forceinline__ void compact_refs(const Compact& c, int id, int total) {
    c.refs_out[id] = id >= total ? 0 : c.was[id] > 0 ? c.was[id] : c.was[c.pairs[c.place[id]].x];
}

__device__ __forceinline__ void compact_row(const Compact& c, int s, int lane, int total) {
    const int len = c.lens[s], need = need_of(len, c.block_size, c.width);
    const int64_t row = (int64_t)s * c.width;
    uint32_t bad = need < 0 ? (uint32_t)kErrBadLength : 0;
    for (int j = lane; j < c.width; j += 32) {
        int b = c.tables[row + j];
        if (j < need) {
            if (b < 0 || b >= c.nb || c.was[b] <= 0) bad |= kErrBadBlock;
            else if (b >= total) b = c.pairs[c.place[b]].y;
        }
        c.tables_out[row + j] = b;
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    if (bad && lane == 0) atomicOr(reinterpret_cast<uint32_t*>(c.result + 1), bad);
}

__global__ void __launch_bounds__(kChunk) compact_solo_kernel(Compact c, int chunks) {
    extern __shared__ int scratch[];
    __shared__ int counts[kSoloBlocks / kChunk];
    c.counts = counts, c.was = scratch, c.place = scratch + chunks * kChunk;
    grid_wait();
    for (int i = 0; i < chunks; ++i) compact_count(c, i);
    __syncthreads();
    for (int i = 0; i < chunks; ++i) compact_assign(c, i, chunks);
    const int total = sum_of_counts(c.counts, chunks);
    __syncthreads();
    for (int id = threadIdx.x; id < c.nb; id += kChunk) compact_refs(c, id, total);
    for (int s = threadIdx.x >> 5; s < c.num_seqs; s += kChunk / 32) compact_row(c, s, threadIdx.x & 31, total);
}
__global__ void __launch_bounds__(kChunk) compact_count_kernel(Compact c) {
    grid_wait();
    compact_count(c, blockIdx.x);
}
__global__ void __launch_bounds__(kChunk) compact_assign_kernel(Compact c, int chunks) {
    grid_wait();
    compact_assign(c, blockIdx.x, chunks);
}
// Thread blocks below `chunks` write reference counts, the others table rows, 32 each.
__global__ void __launch_bounds__(kChunk) compact_write_kernel(Compact c, int chunks) {
    grid_wait();
    const int total = sum_of_counts(c.counts, chunks);
    if ((int)blockIdx.x < chunks) {
        const int id = blockIdx.x * kChunk + threadIdx.x;
        if (id < c.nb) compact_refs(c, id, total);
    } else {
        const int s = (blockIdx.x - chunks) * (kChunk / 32) + (threadIdx.x >> 5);
        if (s < c.num_seqs) compact_row(c, s, threadIdx.x & 31, total);
    }
}

// ---------------------------------------------------------------------------------------------
// copy
// ---------------------------------------------------------------------------------------------

struct CopyView {  // one rank's pool
    uint64_t base;
    int64_t s_layer, s_kv, s_block;
    int32_t nb, layers;
    uint32_t run_bytes, pieces;  // contiguous bytes; pieces of kPiece that a block (dense) has
    uint32_t runs, n2;           // strided: run r is at (r / n2) * s1 + (r % n2) * s2
    int64_t s1, s2;
};
constexpr int kCopyViews = 40, kCopyThreads = 256;
constexpr uint32_t kPiece = 4096;  // bytes that a warp moves at a time: 8 loads of 16 bytes in flight in each lane
struct CopyArgs {
    CopyView v[kCopyViews];
    const int2* pairs;
    const int32_t* count;
    int32_t max_pairs, views;
};

template <bool DENSE>
__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const __grid_constant__ CopyArgs a) {
    grid_wait();
    const uint32_t n = (uint32_t)min(max(*a.count, 0), a.max_pairs);
    if (n == 0) return;
    const int lane = threadIdx.x & 31;
    const uint64_t warps = (uint64_t)gridDim.x * (kCopyThreads / 32);
    uint64_t at = (uint64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5);
    for (int i = 0; i < a.views; ++i) {
        const CopyView& v = a.v[i];
        const uint64_t of_plane = (uint64_t)n * v.pieces, items = of_plane * 2 * v.layers;
        for (; at < items; at += warps) {
            const uint32_t plane = (uint32_t)(at / of_plane), in = (uint32_t)(at - plane * of_plane);
            const uint32_t pair = in / v.pieces, piece = in - pair * v.pieces;
            const int2 p = a.pairs[pair];
            if (p.x < 0 || p.x >= v.nb || p.y < 0 || p.y >= v.nb) continue;
            const uint64_t base = v.base + (plane >> 1) * v.s_layer + (plane & 1) * v.s_kv;
            const uint64_t src = base + p.x * v.s_block, dst = base + p.y * v.s_block;
            const uint32_t bytes = DENSE ? v.run_bytes : v.run_bytes * v.runs;
            const uint32_t first = piece * kPiece + lane * 16;
            uint4 x[8];
            uint64_t off[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t b = first + u * 512;
                if (DENSE) {
                    off[u] = b;
                } else {
                    const uint32_t r = b / v.run_bytes;
                    off[u] = (r / v.n2) * v.s1 + (r % v.n2) * v.s2 + (b - r * v.run_bytes);
                }
                if (b < bytes)
                    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(x[u].x), "=r"(x[u].y), "=r"(x[u].z), "=r"(x[u].w) : "l"(src + off[u]));
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (first + u * 512 < bytes)
                    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(dst + off[u]), "r"(x[u].x), "r"(x[u].y),
                                 "r"(x[u].z), "r"(x[u].w) : "memory");
        }
        at -= items;
    }
}

// Scratch of `ints` words from the library's pool, for the work that `use` enqueues on the stream.
template <class Use>
remp_status with_scratch(int64_t ints, cudaStream_t stream, const Use& use) {
    int device = -1;
    REMP_CUDA(cudaGetDevice(&device));
    cudaMemPool_t pool = nullptr;
    if (remp_status st = device_pool(device, &pool)) return st;
    void* p = nullptr;
    REMP_CUDA(cudaMallocFromPoolAsync(&p, (size_t)ints * 4, pool, stream));
    const cudaError_t e = use(static_cast<int*>(p));
    cudaFreeAsync(p, stream);
    return e == cudaSuccess ? REMP_OK : cuda_fail(e, "page tables");
}

remp_status check_tables(const void* lens, const void* tables, int32_t num_seqs, int32_t width, int32_t block_size,
                         const void* refs, const void* refs_out, int32_t num_blocks, const void* result) {
    if (num_seqs < 0 || width < 0 || num_blocks < 0) return fail(REMP_ERR_INVALID_ARG, "negative dimensions");
    if (block_size < 1) return fail(REMP_ERR_SHAPE, "block_size must be positive");
    if ((num_seqs > 0 && (!lens || (width > 0 && !tables))) || (num_blocks > 0 && (!refs || !refs_out)) || !result)
        return fail(REMP_ERR_INVALID_ARG, "null argument");
    if ((int64_t)num_seqs + 256 > 0x7fffffffLL || (int64_t)num_blocks + kChunk > 0x7fffffffLL)
        return fail(REMP_ERR_SHAPE, "too many sequences or blocks");
    return REMP_OK;
}

}  // namespace

}  // namespace remp

using namespace remp;

extern "C" remp_status remp_pages_fork(int32_t* seq_lens, int32_t* block_tables, int32_t num_seqs,
                                       int32_t max_blocks_per_seq, int32_t block_size, const int32_t* parents,
                                       const int32_t* children, int32_t num_forks, const int32_t* refs,
                                       int32_t* refs_out, int32_t num_blocks, int32_t* pairs, int32_t* result,
                                       void* stream_) {
    if (remp_status st = check_tables(seq_lens, block_tables, num_seqs, max_blocks_per_seq, block_size, refs, refs_out, num_blocks, result))
        return st;
    if (num_forks < 0 || num_forks > 0x7ffffc00) return fail(REMP_ERR_INVALID_ARG, "bad number of children");
    if (num_forks > 0 && (!parents || !children || !pairs)) return fail(REMP_ERR_INVALID_ARG, "null argument");
    if (reinterpret_cast<uint64_t>(pairs) & 7) return fail(REMP_ERR_SHAPE, "pairs must be 8-byte aligned");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    Fork f{seq_lens, block_tables, num_seqs, max_blocks_per_seq, block_size, parents, children, num_forks, refs, refs_out, num_blocks,
           reinterpret_cast<int2*>(pairs), result, nullptr, nullptr, nullptr, nullptr};
    const int chunks = std::max(1, (num_blocks + kChunk - 1) / kChunk);
    if (num_blocks <= kSoloBlocks && num_forks <= kSoloForks && (int64_t)num_forks * max_blocks_per_seq <= kSoloEntries) {
        REMP_CUDA(launch_after(fork_solo_kernel, 1, kChunk, 0, stream, f, chunks));
        return REMP_OK;
    }
    return with_scratch((int64_t)chunks + 2 * (int64_t)num_forks + 3, stream, [&](int* p) {
        f.counts = p, f.nth = p + chunks, f.ids = f.nth + num_forks, f.words = f.ids + num_forks;
        cudaError_t e = launch_after(fork_count_kernel, (int64_t)chunks + 1, kChunk, 0, stream, f, chunks);
        if (e == cudaSuccess) e = launch_after(fork_ids_kernel, chunks, kChunk, 0, stream, f, chunks);
        if (e == cudaSuccess && num_forks > 0) e = launch_after(fork_rows_kernel, ((int64_t)num_forks + 7) / 8, 256, 0, stream, f);
        return e;
    });
}

extern "C" remp_status remp_pages_free(const int32_t* seq_lens, const int32_t* block_tables, int32_t num_seqs,
                                       int32_t max_blocks_per_seq, int32_t block_size, const int32_t* finished,
                                       const int32_t* refs, int32_t num_blocks, int32_t* seq_lens_out,
                                       int32_t* block_tables_out, int32_t* refs_out, int32_t* result, void* stream_) {
    if (remp_status st = check_tables(seq_lens, block_tables, num_seqs, max_blocks_per_seq, block_size, refs, refs_out, num_blocks, result))
        return st;
    if (num_seqs > 0 && (!finished || !seq_lens_out || (max_blocks_per_seq > 0 && !block_tables_out)))
        return fail(REMP_ERR_INVALID_ARG, "null argument");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const Free f{seq_lens, block_tables, num_seqs, max_blocks_per_seq, block_size, finished, refs, num_blocks, seq_lens_out,
                 block_tables_out, refs_out, result};
    if (num_blocks <= kSoloBlocks && (int64_t)num_seqs * std::max(max_blocks_per_seq, 32) <= kSoloEntries) {
        REMP_CUDA(launch_after(free_solo_kernel, 1, kChunk, 0, stream, f));
        return REMP_OK;
    }
    REMP_CUDA(launch_after(free_begin_kernel, std::min<int64_t>(592, num_blocks / 256 + 1), 256, 0, stream, f));
    if (num_seqs > 0) REMP_CUDA(launch_after(free_rows_kernel, ((int64_t)num_seqs + 7) / 8, 256, 0, stream, f));
    return REMP_OK;
}

extern "C" remp_status remp_pages_compact(const int32_t* seq_lens, const int32_t* block_tables, int32_t num_seqs,
                                          int32_t max_blocks_per_seq, int32_t block_size, const int32_t* refs,
                                          int32_t num_blocks, int32_t* block_tables_out, int32_t* refs_out,
                                          int32_t* pairs, int32_t max_pairs, int32_t* result, void* stream_) {
    if (remp_status st = check_tables(seq_lens, block_tables, num_seqs, max_blocks_per_seq, block_size, refs, refs_out, num_blocks, result))
        return st;
    if (num_seqs > 0 && max_blocks_per_seq > 0 && !block_tables_out) return fail(REMP_ERR_INVALID_ARG, "null argument");
    if (max_pairs < num_blocks / 2 || (max_pairs > 0 && !pairs))
        return fail(REMP_ERR_INVALID_ARG, "pairs must have num_blocks / 2 rows");
    if (max_pairs > 0x7fffffff - kChunk) return fail(REMP_ERR_SHAPE, "too many rows of pairs");
    if (reinterpret_cast<uint64_t>(pairs) & 7) return fail(REMP_ERR_SHAPE, "pairs must be 8-byte aligned");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    Compact c{seq_lens, block_tables, num_seqs, max_blocks_per_seq, block_size, refs, num_blocks, block_tables_out, refs_out,
              reinterpret_cast<int2*>(pairs), max_pairs, result, nullptr, nullptr, nullptr};
    const int chunks = std::max(1, (num_blocks + kChunk - 1) / kChunk);
    if (num_blocks <= kSoloBlocks && (int64_t)num_seqs * std::max(max_blocks_per_seq, 32) <= kSoloEntries) {
        const size_t smem = (size_t)2 * chunks * kChunk * 4;
        REMP_CUDA(launch_after(compact_solo_kernel, 1, kChunk, smem, stream, c, chunks));
        return REMP_OK;
    }
    return with_scratch((int64_t)chunks + 2 * (int64_t)num_blocks, stream, [&](int* p) {
        c.counts = p, c.was = p + chunks, c.place = c.was + num_blocks;
        cudaError_t e = launch_after(compact_count_kernel, chunks, kChunk, 0, stream, c);
        if (e == cudaSuccess) e = launch_after(compact_assign_kernel, chunks, kChunk, 0, stream, c, chunks);
        const int64_t rows = ((int64_t)num_seqs + kChunk / 32 - 1) / (kChunk / 32);
        if (e == cudaSuccess) e = launch_after(compact_write_kernel, chunks + rows, kChunk, 0, stream, c, chunks);
        return e;
    });
}

extern "C" remp_status remp_pages_copy(const remp_topo* topo, const remp_model_shape* shape, const remp_shard* shards,
                                       const int32_t* pairs, const int32_t* count, int32_t max_pairs, void* stream_) {
    if (!topo || !shape || !shards || !count || max_pairs < 0 || (max_pairs > 0 && !pairs))
        return fail(REMP_ERR_INVALID_ARG, "null argument or negative max_pairs");
    if (reinterpret_cast<uint64_t>(pairs) & 7) return fail(REMP_ERR_SHAPE, "pairs must be 8-byte aligned");
    const remp_model_shape& m = *shape;
    if (remp_status st = check_shape(m)) return st;
    TopoMap T;
    std::string why;
    if (remp_status st = build_topo_map(*topo, m, &T, &why)) return fail(st, why);
    const int64_t row = (int64_t)m.head_dim * m.elem_bytes, slice = row * m.block_size;
    std::vector<CopyView> views;
    bool dense = true;
    for (int r = 0; r < T.num_ranks(); ++r) {
        ShardView s;
        const int layers = T.stage_layers(r / T.tp), heads = T.heads_per_rank;
        if (remp_status st = resolve_shard(shards[r], T, layers, m, &s)) return st;
        if (s.nb > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "block ids are 32-bit");
        CopyView v{s.base, s.s_layer, s.s_kv, s.s_block, (int32_t)s.nb, layers, 0, 0, 1, 1, 0, 0};
        if (s.s_token == row && (s.s_head == slice || heads == 1)) {
            v.run_bytes = (uint32_t)(heads * slice);  // head-major, dense
        } else if (s.s_head == row && s.s_token == heads * row) {
            v.run_bytes = (uint32_t)(heads * slice);  // token-major, dense
        } else if (s.s_token == row) {
            if (s.s_head < slice) return fail(REMP_ERR_SHAPE, "stride_head must hold a head slice");
            v.run_bytes = (uint32_t)slice, v.runs = (uint32_t)heads, v.n2 = (uint32_t)heads, v.s2 = s.s_head, dense = false;
        } else {
            if (row & 15) return fail(REMP_ERR_SHAPE, "strided token rows must be multiples of 16 bytes");
            v.run_bytes = (uint32_t)row, v.runs = (uint32_t)(heads * m.block_size), v.n2 = (uint32_t)m.block_size;
            v.s1 = s.s_head, v.s2 = s.s_token, dense = false;
        }
        v.pieces = (v.run_bytes * v.runs + kPiece - 1) / kPiece;
        if (layers > 0 && s.nb > 0) views.push_back(v);
    }
    if (max_pairs == 0 || views.empty()) return REMP_OK;
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    for (size_t at = 0; at < views.size(); at += kCopyViews) {  // 40 ranks to a launch
        CopyArgs a{};
        a.views = (int32_t)std::min<size_t>(kCopyViews, views.size() - at);
        int64_t items = 0;
        for (int i = 0; i < a.views; ++i) {
            a.v[i] = views[at + (size_t)i];
            if ((int64_t)max_pairs * a.v[i].pieces > 0xffffffffLL) return fail(REMP_ERR_SHAPE, "too many pairs for one call");
            items += (int64_t)max_pairs * a.v[i].pieces * 2 * a.v[i].layers;
        }
        a.pairs = reinterpret_cast<const int2*>(pairs), a.count = count, a.max_pairs = max_pairs;
        const int64_t grid = std::min<int64_t>((int64_t)sms * 5, (items + kCopyThreads / 32 - 1) / (kCopyThreads / 32));
        REMP_CUDA(launch_after(dense ? pages_copy_kernel<true> : pages_copy_kernel<false>, grid, kCopyThreads, 0, stream, a));
    }
    return REMP_OK;
}
