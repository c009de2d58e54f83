// A cache of 16-bit values as bulk tensor copies bring it to shared memory, a tile of a head at a time.
#pragma once

#include <cuda.h>

#include "remp_kv.h"
#include "remp_tensor.h"

namespace remp {

struct KvBoxes {
    CUtensorMap k, v;         // in boxes of a tile: [slice of a block and head][8 tokens][64 dims][token][dim]
    int32_t i_block, i_head;  // from the slice of a block, of a head to the next
};

// remp_kv.cu. Caches that it cannot state (strides of 2^40 bytes, 2^31 slices) are not taken.
bool kv_boxes_take(const KvView& v);
cudaError_t kv_boxes(const KvView& v, int32_t head_dim, bool bf, KvBoxes* boxes);

#ifdef __CUDACC__

// A tile of a head to `dst`: 8 rows of 128 bytes whose 16-byte pieces change places, of each 64 dims, of each 8 tokens; its bytes
// count for `bar`.
__device__ __forceinline__ void bring_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int eighth, int slice) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %3, %3, %4, %5}], [%2];" ::"r"(dst), "l"(map), "r"(bar),
                 "r"(0), "r"(eighth), "r"(slice)
                 : "memory");
}
// What descriptors of such keys have on top: 8 keys of all dims lie `eight` bytes before the next 8.
__host__ __device__ constexpr uint64_t keys_apart(int eight) { return (uint64_t)(eight - 1024 >> 4) << 32; }

#endif

}  // namespace remp
