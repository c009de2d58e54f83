// What the kernels of attention over a cache of 16-bit values take.
#pragma once

#include "remp_kv.h"

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

}  // namespace remp
