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

// Two probabilities as two numbers of the cache's type each: the first bits, rounded towards 0, and what is left, so that neither
// is below 0; what is left of one above 0 is at least the type's least normal number (bfloat16: 2^-95 of a row's largest and less) or
// its least number (half: 2^-34). With an infinity in V two numbers above 0 give that infinity, 0 would give NaN.
template <bool BF>
__device__ __forceinline__ void split2(float x, float y, uint32_t* high, uint32_t* low) {
    constexpr float kLeast = BF ? 0x1p-126f : 0x1p-24f;
    float2 f;
    if (BF) {
        *high = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
        f = make_float2(bf_low(*high), bf_high(*high));
    } else {
        asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(*high) : "f"(y), "f"(x));
        f = __half22float2(*reinterpret_cast<const __half2*>(high));
    }
    *low = pack2(fmaxf(x - f.x, fminf(x, kLeast)), fmaxf(y - f.y, fminf(y, kLeast)), BF);
}

#endif

}  // namespace remp
