// Rows of new tokens on their way into a cache: what is done to them, and 16-bit values to 32 bits and back.
#pragma once

#include "remp_kvq.h"

namespace remp {

struct Transform {
    const float* q_norm;
    const float* k_norm;
    const float* rope;
    const int32_t* positions;
    float eps;
    int32_t rope_rows, rotary_dim, interleaved;
};

// The caller's transform, checked (NULL: neither norm nor rotation); remp_kvq.cu.
remp_status kvq_transform(const remp_kvq_transform* transform, int32_t head_dim, Transform* tr);

#ifdef __CUDACC__

template <bool BF>
__device__ __forceinline__ void unpack8(const uint4& raw, float (&x)[8]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF) {
            x[2 * i] = bf_low(w[i]), x[2 * i + 1] = bf_high(w[i]);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}

template <bool BF>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

#endif

}  // namespace remp
