// What the kernels of attention over a cache of 16-bit values take.
#pragma once

#include "remp_kv.h"
#include "remp_kvq_device.h"

namespace remp {

struct KvAttendArgs {
    KvView v;
    KvqRows q, out;
    float* lse;
    uint8_t* workspace;
    float scale_log2;  // softmax scale * log2(e)
    int32_t group, q_heads, window, first;
    uint32_t by_group; // row / group = high half of row * by_group (0: group is 1)
    int32_t room;      // tokens that a row of the table holds
};

// remp_kv_prompt.cu: many queries of a sequence, of a cache that comes in boxes
cudaError_t launch_kv_prompt(const KvAttendArgs& a, int32_t head_dim, bool bf, int sms, int32_t max_rows, cudaStream_t stream);

#ifdef __CUDACC__

// Two probabilities as two numbers of the cache's type each: the first bits, rounded towards 0, and what is left of them, so that
// neither is below 0. What is left of one above 0 is not 0 either: with an infinity in V, two numbers above 0 give that infinity, 0
// would give NaN. bfloat16: the last of a probability's 24 bits is set, so 2^-23 of it are left at least (enough from 2^-72 of a row's
// largest on). Half: it is the type's least number at least, 2^-32 of a row's largest.
template <bool BF>
__device__ __forceinline__ uint32_t first2(float x, float y) {
    if (BF) return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
    uint32_t r;
    asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}
template <bool BF>
__device__ __forceinline__ uint32_t left2(float x, float y, uint32_t first) {
    if (BF) return pack2(__uint_as_float(__float_as_uint(x) | 1) - bf_low(first), __uint_as_float(__float_as_uint(y) | 1) - bf_high(first), true);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&first));
    return pack2(fmaxf(x - f.x, fminf(x, 0x1p-24f)), fmaxf(y - f.y, fminf(y, 0x1p-24f)), false);
}

#endif

}  // namespace remp
