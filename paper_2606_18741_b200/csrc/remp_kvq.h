// The 4-bit cache as its kernels see it (format: include/remp.h), and what they share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "remp_internal.h"
#include "remp_kvq_span.h"

namespace remp {

constexpr int kKvqGroup = 64;  // dims that share a step and a minimum
constexpr int kKvqTile = 16;   // tokens of a tile

__host__ __device__ constexpr int kvq_token_bytes(int d) { return d / 2 + d / 16; }

struct KvqView {           // one layer of a rank's pool, strides in bytes
    uint8_t* base;         // K of block 0, head 0 in the layer
    int64_t s_kv, s_block, s_head;
    int32_t nb;            // blocks
    int32_t kv_heads;
    int32_t block_tiles;   // block_size / 16
    int32_t max_blocks, num_seqs, num_tokens;
    const int32_t* seq_lens;
    const int32_t* tables;
    const int32_t* query_start;
    uint32_t* error;
};

struct KvqRows {  // strides in elements
    uint16_t* data;
    int64_t s_token, s_head;
};

// Checks of what every call on the cache takes; remp_kvq.cu.
remp_status kvq_view(const remp_kvq_pool* pool, const remp_kvq_batch* batch, KvqView* v);
// Strides of a single head or token are whatever the caller's tensor says; inputs may repeat a row (stride 0), outputs may not.
remp_status kvq_rows(const remp_kvq_rows* r, int32_t tokens, int32_t heads, int32_t head_dim, bool written, const char* name, KvqRows* out);

#ifdef __CUDACC__

__device__ __forceinline__ float bf_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ void kvq_error(const KvqView& v, uint32_t bit) {
    if (v.error) atomicOr(v.error, bit);
}

// The sequence that row t belongs to: the last s with query_start[s] <= t. A warp looks at 32 places at a time, so 1024
// sequences take two dependent loads instead of ten. -1: none (t before query_start[0]).
__device__ __forceinline__ int kvq_sequence_of(const KvqView& v, int t) {
    int lo = 0, n = v.num_seqs;  // the answer is in [lo - 1, lo + n)
    const int lane = threadIdx.x & 31;
    while (n > 0) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const bool below = lane * step < n && v.query_start[at] <= t;
        const unsigned votes = __ballot_sync(0xffffffffu, below);
        if (!votes) return lo - 1;
        const int last = 31 - __clz(votes);
        const int end = lo + n;
        lo += last * step + 1;
        n = min(step - 1, end - lo);
    }
    return lo - 1;
}

#endif

}  // namespace remp
