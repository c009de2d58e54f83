// Writing a cache of 16-bit values (rules: include/remp.h), and the checks that all calls on it share.
//
// Mathematics, per row x of one head of one token: xn = x / sqrt(mean(x^2) + eps) * w, then pairs (a, b) of dims turn to
// (a cos - b sin, b cos + a sin), in 32 bits, rounded once to 16. Values are copied.
//
// Bound: HBM, each row is read and written once. A row is held by head_dim/8 lanes, 8 dims (16 bytes) each: the norm is a butterfly over
// these lanes, a turn's partner dim is in the same lane (interleaved) or one shuffle away. A warp takes the rows of ONE
// token, kSets sets at a time: it looks up where the token belongs and loads its cosines and sines once, and asks for the
// next sets' rows before this one's are worked on. Where tokens are too few to fill the GPU that way, every kSets sets get a
// warp of their own. Sets are four at a time there (the fewest steps: 6 us for 256 tokens of 80 heads, 8 us with two), and two else,
// which leaves room for seven thread blocks on an SM instead of five: norms keep the issue slots busy, and waits need more warps
// to fill them (31 900 tokens of 40 heads: 150 us, from 172, and 123 with one instruction for the root and its reciprocal).

#include "remp_kv.h"

#include <algorithm>
#include <numeric>

#include "remp_kv_boxes.h"
#include "remp_rows.h"

namespace remp {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

struct Slot {  // where a token's rows are
    int64_t off;   // bytes from the pool's base to its row of head 0, K
    int32_t pos;   // position in its sequence
    bool known;    // the token has a position
    bool stored;   // and a block
};

// The slot of row `token`; a whole warp asks for the same token.
__device__ __forceinline__ Slot find_slot(const KvView& v, int token) {
    Slot r{0, -1, false, false};
    const int s = kvq_sequence_of(v, token);
    if (s < 0) return r;
    const int end = v.query_start[s + 1];
    if (token >= end) return r;
    const int64_t pos = (int64_t)v.seq_lens[s] - end + token;
    const int64_t tile = pos >> 4;
    if (pos < 0 || tile >= (int64_t)v.max_blocks * v.block_tiles) return r;
    r.pos = (int)pos, r.known = true;
    const int in_row = (int)tile / v.block_tiles;
    const int block = v.tables[(int64_t)s * v.max_blocks + in_row];
    r.stored = block >= 0 && block < v.nb;
    r.off = (int64_t)block * v.s_block + (int64_t)((int)pos - in_row * v.block_tiles * kKvqTile) * v.s_token;
    return r;
}

struct Turn {  // cosines and sines of a lane's dims, the sines with the sign of their product; partner lane of pairs half a row apart
    float cs[8], sn[8];
    int partner;
    bool here, interleaved, any;
};

// Norm and turn of a row's 8 dims in this lane; all lanes of the row are here.
template <int D, bool BF>
__device__ __forceinline__ uint4 turned(const uint4& raw, const float* norm, float eps, const Turn& t, int l) {
    if (!norm && !t.any) return raw;
    float x[8];
    unpack8<BF>(raw, x);
    if (norm) {
        float sum = ((x[0] * x[0] + x[1] * x[1]) + (x[2] * x[2] + x[3] * x[3])) + ((x[4] * x[4] + x[5] * x[5]) + (x[6] * x[6] + x[7] * x[7]));
#pragma unroll
        for (int s = 1; s < D / 8; s <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
        const float r = rsqrtf(fmaf(sum, 1.f / D, eps));  // off by 2^-22; the row is rounded to 2^-12 of itself at best
        const float4 a = __ldg(reinterpret_cast<const float4*>(norm + 8 * l)), b = __ldg(reinterpret_cast<const float4*>(norm + 8 * l + 4));
        const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
    }
    if (t.any && t.interleaved) {
        if (t.here) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = fmaf(a, t.cs[i], -b * t.sn[i]);
                x[2 * i + 1] = fmaf(b, t.cs[i], a * t.sn[i]);
            }
        }
    } else if (t.any) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl_sync(0xffffffffu, x[i], t.partner);
            if (t.here) x[i] = fmaf(x[i], t.cs[i], other * t.sn[i]);
        }
    }
    return pack8<BF>(x);
}

// The work is in groups of kSets sets of rows: a token's groups of query heads, then of K, then of V; a warp takes
// `per_warp` groups of one token.
template <int D, bool BF, int kSets>
__global__ void __launch_bounds__(kThreads, kSets == 4 ? 5 : 7) kv_append_kernel(const KvView v, const KvqRows q, const KvqRows k, const KvqRows val,
                                                               const KvqRows q_out, const Transform tr, const int q_heads,
                                                               const int q_groups, const int kv_groups, const int per_warp) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kStep = kSets * kRows;  // lanes of a row, rows of a warp, heads of a group
    grid_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const int groups = q_groups + 2 * kv_groups, shares = (groups + per_warp - 1) / per_warp;
    const int64_t all = (int64_t)v.num_tokens * shares, step_of_grid = (int64_t)gridDim.x * kWarps;

    for (int64_t share = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); share < all; share += step_of_grid) {
        const int token = (int)(share / shares), begin = (int)(share - (int64_t)token * shares) * per_warp;
        const int end = min(groups, begin + per_warp);
        const auto load = [&](int group, uint4 (&raw)[kSets]) {
            const bool of_q = group < q_groups, of_v = group >= q_groups + kv_groups;
            const KvqRows& from = of_q ? q : of_v ? val : k;
            const int heads = of_q ? q_heads : v.kv_heads, head0 = (of_q ? group : of_v ? group - q_groups - kv_groups : group - q_groups) * kStep + sub;
            const uint16_t* p = from.data + token * from.s_token + head0 * from.s_head + 8 * l;
            const int64_t step = kRows * from.s_head;
#pragma unroll
            for (int u = 0; u < kSets; ++u) raw[u] = head0 + u * kRows < heads ? *reinterpret_cast<const uint4*>(p + u * step) : make_uint4(0, 0, 0, 0);
        };
        uint4 raw[kSets];
        load(begin, raw);

        const Slot slot = find_slot(v, token);
        bool known = slot.known;
        int rope_row = slot.pos;
        if (tr.rope && known) {
            if (tr.positions) rope_row = tr.positions[token];
            known = rope_row >= 0 && rope_row < tr.rope_rows;
        }
        if (!known || !slot.stored) {
            if (lane == 0) kvq_error(v, known ? kErrBadBlock : kErrBadLength);
            if (!known) continue;
        }
        Turn turn;
        const int half = tr.rotary_dim / 2;
        turn.any = tr.rope != nullptr, turn.here = tr.rope && 8 * l < tr.rotary_dim, turn.interleaved = tr.interleaved, turn.partner = lane;
        if (turn.here) {
            const float* row = tr.rope + (int64_t)rope_row * tr.rotary_dim;
            if (tr.interleaved) {
                const float4 c = *reinterpret_cast<const float4*>(row + 4 * l);
                const float4 s = *reinterpret_cast<const float4*>(row + half + 4 * l);
                turn.cs[0] = c.x, turn.cs[1] = c.y, turn.cs[2] = c.z, turn.cs[3] = c.w, turn.sn[0] = s.x, turn.sn[1] = s.y, turn.sn[2] = s.z, turn.sn[3] = s.w;
            } else {
                const bool upper = 8 * l >= half;
                const float* c = row + 8 * l - (upper ? half : 0);
                const float sign = upper ? 1.f : -1.f;
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 a = *reinterpret_cast<const float4*>(c + i), b = *reinterpret_cast<const float4*>(c + half + i);
                    turn.cs[i] = a.x, turn.cs[i + 1] = a.y, turn.cs[i + 2] = a.z, turn.cs[i + 3] = a.w;
                    turn.sn[i] = b.x * sign, turn.sn[i + 1] = b.y * sign, turn.sn[i + 2] = b.z * sign, turn.sn[i + 3] = b.w * sign;
                }
                turn.partner = lane + (upper ? -half / 8 : half / 8);
            }
        }
        uint8_t* const row0 = v.base + slot.off + 16 * l;

#pragma unroll 1
        for (int group = begin; group < end; ++group) {
            uint4 now[kSets];
#pragma unroll
            for (int u = 0; u < kSets; ++u) now[u] = raw[u];
            if (group + 1 < end) load(group + 1, raw);
            if (group < q_groups) {
                const int head0 = group * kStep + sub;
                uint16_t* p = q_out.data + token * q_out.s_token + head0 * q_out.s_head + 8 * l;
#pragma unroll
                for (int u = 0; u < kSets; ++u) {
                    const uint4 x = turned<D, BF>(now[u], tr.q_norm, tr.eps, turn, l);
                    if (head0 + u * kRows < q_heads) *reinterpret_cast<uint4*>(p + u * kRows * q_out.s_head) = x;
                }
            } else {
                const bool of_v = group >= q_groups + kv_groups;
                const int head0 = (group - q_groups - (of_v ? kv_groups : 0)) * kStep + sub;
                uint8_t* p = row0 + head0 * v.s_head + (of_v ? v.s_kv : 0);
#pragma unroll
                for (int u = 0; u < kSets; ++u) {
                    const uint4 x = of_v ? now[u] : turned<D, BF>(now[u], tr.k_norm, tr.eps, turn, l);
                    if (slot.stored && head0 + u * kRows < v.kv_heads) *reinterpret_cast<uint4*>(p + u * kRows * v.s_head) = x;
                }
            }
        }
    }
}

template <int D, bool BF>
auto append_kernel(bool few) { return few ? kv_append_kernel<D, BF, 4> : kv_append_kernel<D, BF, 2>; }

}  // namespace

remp_status kv_pool_view(const remp_kv_pool* pool, KvView* v) {
    if (!pool) return fail(REMP_ERR_INVALID_ARG, "null pool");
    if (pool->head_dim != 64 && pool->head_dim != 128 && pool->head_dim != 256)
        return fail(REMP_ERR_SHAPE, "head_dim of a 16-bit cache must be 64, 128 or 256");
    if (pool->block_size < kKvqTile || pool->block_size % kKvqTile)
        return fail(REMP_ERR_SHAPE, "block_size must be a multiple of 16");
    if (pool->kv_heads < 1) return fail(REMP_ERR_SHAPE, "kv_heads must be positive");
    if (pool->layer < 0) return fail(REMP_ERR_INVALID_ARG, "negative layer");
    const remp_model_shape m = {1, pool->kv_heads, pool->head_dim, pool->block_size, 2};
    TopoMap T;
    T.heads_per_rank = pool->kv_heads;
    ShardView s;
    if (remp_status st = resolve_shard(pool->shard, T, 1, m, &s)) return st;
    const int64_t row = 2 * (int64_t)pool->head_dim, last_token = (pool->block_size - 1) * s.s_token, last_head = (pool->kv_heads - 1) * s.s_head;
    if (pool->kv_heads > 1 && s.s_head < last_token + row && s.s_token < last_head + row)
        return fail(REMP_ERR_SHAPE, "stride_head must hold a head's tokens, or stride_token a token's heads");
    if (s.nb > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "block ids are 32-bit");
    *v = KvView{};
    v->base = reinterpret_cast<uint8_t*>(s.base + (uint64_t)((int64_t)pool->layer * s.s_layer));
    v->s_kv = s.s_kv, v->s_block = s.s_block, v->s_head = s.s_head, v->s_token = s.s_token;
    v->nb = (int32_t)s.nb, v->kv_heads = pool->kv_heads, v->block_tiles = pool->block_size / kKvqTile;
    return REMP_OK;
}

remp_status kv_view(const remp_kv_pool* pool, const remp_kvq_batch* batch, KvView* v) {
    if (!pool || !batch) return fail(REMP_ERR_INVALID_ARG, "null pool or batch");
    if (remp_status st = kv_pool_view(pool, v)) return st;
    return kvq_batch_view(batch, v);
}

remp_status kv_mask(float scale, int32_t window, int32_t first) {
    if (window < 0 || first < 0) return fail(REMP_ERR_INVALID_ARG, "negative window or number of first tokens");
    if (!(scale > 0.f && scale <= 3.402823466e38f)) return fail(REMP_ERR_INVALID_ARG, "scale must be positive and finite");
    return REMP_OK;
}

remp_status kv_group(int32_t q_heads, int32_t kv_heads, int64_t num_tokens, int32_t* group, uint32_t* by_group) {
    if (q_heads < 1 || q_heads % kv_heads) return fail(REMP_ERR_SHAPE, "q_heads must be a multiple of kv_heads");
    const int32_t g = q_heads / kv_heads;
    if (g > 0x8000 || num_tokens * g * g > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "too many query rows");
    *group = g, *by_group = g == 1 ? 0 : (uint32_t)((0x100000000ULL + g - 1) / g);
    return REMP_OK;
}

namespace {

// Blocks and heads as one dimension of a tensor map: slices at the largest step that meets the heads of all blocks.
struct Slices {
    int64_t step, i_block, i_head, count;
};
Slices slices_of(const KvView& v) {
    int64_t step = 0;
    if (v.nb > 1) step = std::gcd(step, v.s_block);
    if (v.kv_heads > 1) step = std::gcd(step, v.s_head);
    if (step == 0) step = 16;  // a single slice
    Slices s{step, v.nb > 1 ? v.s_block / step : 0, v.kv_heads > 1 ? v.s_head / step : 0, 0};
    s.count = (v.nb - 1) * s.i_block + (v.kv_heads - 1) * s.i_head + 1;
    return s;
}

}  // namespace

bool kv_boxes_take(const KvView& v) {
    // strides and coordinates of a tensor map
    return v.nb > 0 && std::max(8 * v.s_token, std::max(v.s_head, v.s_block)) < (int64_t)1 << 40 && slices_of(v).count <= 0x7fffffff;
}

cudaError_t kv_boxes(const KvView& v, int32_t head_dim, bool bf, KvBoxes* boxes) {
    using Encode = decltype(&cuTensorMapEncodeTiled);
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) == cudaSuccess ? reinterpret_cast<Encode>(f) : nullptr;
    }();
    if (!encode) return cudaErrorNotSupported;
    const Slices s = slices_of(v);
    boxes->i_block = (int32_t)s.i_block, boxes->i_head = (int32_t)s.i_head;
    const cuuint64_t dims[5] = {64, 8, (cuuint64_t)head_dim / 64, (cuuint64_t)v.block_tiles * (kKvqTile / 8), (cuuint64_t)s.count};
    const cuuint64_t strides[4] = {(cuuint64_t)v.s_token, 128, (cuuint64_t)(8 * v.s_token), (cuuint64_t)s.step};
    const cuuint32_t box[5] = {64, 8, (cuuint32_t)head_dim / 64, kKvqTile / 8, 1}, steps[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < 2; ++i)
        if (encode(i ? &boxes->v : &boxes->k, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5, v.base + (i ? v.s_kv : 0), dims, strides, box, steps,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    return cudaSuccess;
}

}  // namespace remp

using namespace remp;

extern "C" remp_status remp_kv_append(const remp_kv_pool* pool, const remp_kvq_batch* batch, const remp_kvq_rows* q,
                                      const remp_kvq_rows* k, const remp_kvq_rows* v, const remp_kvq_rows* q_out,
                                      int32_t q_heads, int32_t dtype, const remp_kvq_transform* transform, void* stream_) {
    KvView view;
    KvqRows rq{nullptr, 0, 0}, rk, rv, ro{nullptr, 0, 0};
    if (remp_status st = kv_view(pool, batch, &view)) return st;
    if (remp_status st = kvq_dtype(dtype)) return st;
    const int32_t d = pool->head_dim;
    if (q_heads < 0 || (q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr))
        return fail(REMP_ERR_INVALID_ARG, "q, q_out and q_heads go together");
    Transform tr;
    if (remp_status st = kvq_transform(transform, d, &tr)) return st;
    if (view.num_tokens == 0) return REMP_OK;
    if (q_heads) {
        if (remp_status st = kvq_rows(q, view.num_tokens, q_heads, d, false, "q", &rq)) return st;
        if (remp_status st = kvq_rows(q_out, view.num_tokens, q_heads, d, true, "q_out", &ro)) return st;
    }
    if (remp_status st = kvq_rows(k, view.num_tokens, pool->kv_heads, d, false, "k", &rk)) return st;
    if (remp_status st = kvq_rows(v, view.num_tokens, pool->kv_heads, d, false, "v", &rv)) return st;
    const int64_t rows = (int64_t)q_heads + 2 * (int64_t)pool->kv_heads;
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    // Few tokens: a warp to a group of four sets; many: a token to a warp. Both, us in a graph, for 1000, 2000 and 5000 tokens: 64 + 2 x 8
    // heads of 128 dims 18 and 23, 29 and 27, 57 and 51; 32 + 2 x 4 with norms 16 and 16, 25 and 18, 45 and 33; 32 + 2 x 8 of 64 dims
    // 12 and 12, 16 and 14, 29 and 21; 16 + 2 x 2 of 256 14 and 14, 20 and 16, 39 and 31; 300 tokens of these: 8 to 10 and 12 to 20.
    const bool few = view.num_tokens < sms * 10, bf = dtype == REMP_DTYPE_BFLOAT;
    const int heads = 32 / (d / 8) * (few ? 4 : 2);  // of a group
    if (rows > 0x7fffffffLL - 3 * heads) return fail(REMP_ERR_SHAPE, "too many heads");
    const int q_groups = (q_heads + heads - 1) / heads, kv_groups = (pool->kv_heads + heads - 1) / heads, groups = q_groups + 2 * kv_groups;
    // a token to a warp when that fills the GPU, else a group
    const int per_warp = few ? 1 : groups;
    const int64_t shares = (int64_t)view.num_tokens * ((groups + per_warp - 1) / per_warp);
    const int64_t grid = std::min<int64_t>((shares + kWarps - 1) / kWarps, (int64_t)sms * 48);
    const auto kernel = d == 64    ? (bf ? append_kernel<64, true>(few) : append_kernel<64, false>(few))
                        : d == 128 ? (bf ? append_kernel<128, true>(few) : append_kernel<128, false>(few))
                                   : (bf ? append_kernel<256, true>(few) : append_kernel<256, false>(few));
    REMP_CUDA(launch_after(kernel, grid, kThreads, 0, static_cast<cudaStream_t>(stream_), view, rq, rk, rv, ro, tr, (int)q_heads, q_groups, kv_groups,
                           per_warp));
    return REMP_OK;
}
