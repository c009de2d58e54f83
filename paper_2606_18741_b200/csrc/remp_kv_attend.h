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

// A probability x as two numbers of the cache's type: the first bits, f, rounded towards 0, and what is left of it, so that neither is
// below 0. What is left of one above 0 is not 0 either: with an infinity in V, two numbers above 0 give that infinity, 0 would give
// NaN. In bfloat16 it is x (1 + 2^-22) - f, 2^-22 of x at least (enough from 2^-72 of a row's largest on); in half the type's least
// number at least, 2^-32 of a row's largest.
constexpr float kAndMore = 1.f + 0x1p-22f, kLeastHalf = 0x1p-24f;

#endif

}  // namespace remp
