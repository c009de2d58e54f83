// What the kernels that weigh cached positions take.
#pragma once

#include "remp_kv.h"

namespace remp {

struct WeighArgs {
    KvView v;
    KvqRows q;
    const float* lse;
    float* weights;
    int64_t stride;
    float scale_log2;
    int32_t group, q_heads, window, first, fresh;
    uint32_t by_group;
    int32_t room;  // tokens that a row of the table and a row of the weights hold
};

// remp_kv_weigh_wide.cu: many rows of a sequence, of a cache that comes in boxes
cudaError_t launch_kv_weigh_wide(const WeighArgs& a, int32_t head_dim, bool bf, int sms, cudaStream_t stream);

}  // namespace remp
