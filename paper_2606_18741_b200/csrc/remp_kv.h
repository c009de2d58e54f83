// The cache of 16-bit values as its kernels see it (rules: include/remp.h), and what they share.
#pragma once

#include "remp_kvq.h"
#include "remp_launch.h"

namespace remp {

struct KvView : KvqView {  // a token's row of one head: base + block * s_block + head * s_head + place in the block * s_token, V s_kv behind
    int64_t s_token;
};

// Checks of a pool, and of what the calls with a batch take; remp_kv.cu.
remp_status kv_pool_view(const remp_kv_pool* pool, KvView* v);
remp_status kv_view(const remp_kv_pool* pool, const remp_kvq_batch* batch, KvView* v);
remp_status kv_mask(float scale, int32_t window, int32_t first);
// Rows are divided by the query heads of a KV head with one multiplication, exact while row * group stays below 2^32.
remp_status kv_group(int32_t q_heads, int32_t kv_heads, int64_t num_tokens, int32_t* group, uint32_t* by_group);

#ifdef __CUDACC__

__device__ __forceinline__ int kv_token_of(uint32_t by_group, int row) { return by_group ? (int)__umulhi((uint32_t)row, by_group) : row; }

// d[16][8] += a[16][16] . b[16][8]
template <bool BF>
__device__ __forceinline__ void mma_rows(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

#endif

}  // namespace remp
