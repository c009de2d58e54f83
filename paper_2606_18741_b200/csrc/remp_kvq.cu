// Writing a 4-bit cache and reading it back (format and rules: include/remp.h).
//
// Mathematics, per row x of one head of one token: xn = x / sqrt(mean(x^2) + eps) * w, then pairs (a, b) of dims turn to
// (a cos - b sin, b cos + a sin); queries leave in 16 bits, keys and values as codes c = rint((x - m)/s) with a minimum
// m and a step s for each 64 dims. All sums, norms and turns are in 32 bits; products and sums are rounded one by one
// and the squares are added neighbours first, so that any program that follows the formula in that order gets the same
// codes (a contracted multiply-add would move values on the edge between two codes).
//
// Bound: HBM (each row is read and written once), and issue slots close behind. A row is held by head_dim/8 lanes, 8 dims (16
// bytes) each: the norm is a butterfly over these lanes, a turn's partner dim is in the same lane (interleaved) or one
// shuffle away, and a group of 64 dims is 8 lanes. A warp takes the rows of ONE token, kSets sets at a time: it looks up
// where the token belongs and loads its cosines and sines once, asks for the next sets' rows as soon as this one's are
// unpacked, and takes the square roots and reciprocals of all its sets' norms at once. Where tokens are too few to
// fill the GPU that way, every kSets sets get a warp of their own.
// Measured: 31.9 thousand tokens of 32 + 2 x 4 heads of 128 dims with norms and turns 190 us (585 MB of DRAM traffic, 3.1
// TB/s), bound by issue slots (73 % of them taken); 256 tokens of 64 + 2 x 8 heads 12.7 us. Reading the values of the 31.9
// thousand back 32 us, with the integer pipe at 72 %. All three under a profiler, with a cold cache.

#include <algorithm>

#include "remp_kvq.h"
#include "remp_launch.h"

namespace remp {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kSets = 4;

struct Transform {
    const float* q_norm;
    const float* k_norm;
    const float* rope;
    const int32_t* positions;
    float eps;
    int32_t rope_rows, rotary_dim, interleaved;
};

struct Slot {  // where a token's codes are
    int64_t off;   // bytes from the pool's base to its tile (of head 0, K)
    int32_t pos;   // position in its sequence
    bool known;    // the token has a position
    bool stored;   // and a block
};

// The slot of row `token`; a whole warp asks for the same token.
__device__ __forceinline__ Slot find_slot(const KvqView& v, int token, int tile_bytes) {
    Slot r{0, -1, false, false};
    const int s = kvq_sequence_of(v, token);
    if (s < 0) return r;
    const int end = v.query_start[s + 1];
    if (token >= end) return r;
    const int64_t pos = (int64_t)v.seq_lens[s] - end + token;
    const int64_t tile = pos >> 4;
    if (pos < 0 || tile >= (int64_t)v.max_blocks * v.block_tiles) return r;
    r.pos = (int)pos, r.known = true;
    const int in_row = (int)(tile / v.block_tiles);
    const int block = v.tables[(int64_t)s * v.max_blocks + in_row];
    r.stored = block >= 0 && block < v.nb;
    r.off = (int64_t)block * v.s_block + (int64_t)((int)tile - in_row * v.block_tiles) * tile_bytes;
    return r;
}

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

// One step of a transpose between lanes and nibbles: lane bit `s` changes places with nibble-index bit `s`.
__device__ __forceinline__ uint32_t nibble_step(uint32_t w, int s, uint32_t low, int lane) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, w, s);
    return (lane & s) ? (w & ~low) | ((other & ~low) >> (4 * s)) : (w & low) | ((other & low) << (4 * s));
}

// Codes of 8 neighbouring dims, nibble t + 4e = dim 2t + e (K) or nibble j = dim j (V), to the word that this lane
// stores, and back: both are their own inverse. K: among the four lanes of 32 dims; V: a third step, among the eight of 64.
__device__ __forceinline__ uint32_t k_transpose(uint32_t w, int lane) {
    return nibble_step(nibble_step(w, 1, 0x0f0f0f0fu, lane), 2, 0x00ff00ffu, lane);
}
__device__ __forceinline__ int k_place(int j) { return (j >> 1) + 4 * (j & 1); }

// Byte of lane l's word inside a token's codes.
template <int D>
__device__ __forceinline__ int word_at(int l, bool is_v) {
    return is_v ? (l & 7) * (D / 16) + (l >> 3) * 4 : (l & 3) * (D / 8) + (l >> 2) * 4;
}

struct Turn {  // cosines and sines of a lane's dims, the sines with the sign of their product; partner lane of pairs half a row apart
    float cs[8], sn[8];
    int partner;
    bool here, interleaved, any;
};

// Norm (r: 1 / root mean square) and turn of a row's 8 dims in this lane.
__device__ __forceinline__ void turn_row(float (&x)[8], float r, const float4* weight, const Turn& t) {
    if (weight) {
        const float4 a = weight[0], b = weight[1];
        const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(__fmul_rn(x[i], r), w[i]);
    }
    if (!t.any) return;
    if (t.interleaved) {
        if (t.here) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = __fsub_rn(__fmul_rn(a, t.cs[i]), __fmul_rn(b, t.sn[i]));
                x[2 * i + 1] = __fadd_rn(__fmul_rn(b, t.cs[i]), __fmul_rn(a, t.sn[i]));
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl_sync(0xffffffffu, x[i], t.partner);
            if (t.here) x[i] = __fadd_rn(__fmul_rn(x[i], t.cs[i]), __fmul_rn(other, t.sn[i]));
        }
    }
}

// 1 / root mean square of kSets rows at once: of raw[u]'s in the lanes with lane % 4 = u.
template <int D, bool BF>
__device__ __forceinline__ float row_scales(const uint4 (&raw)[kSets], float eps, int lane) {
    float mean = 0.f;
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        float x[8];
        unpack8<BF>(raw[u], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(x[i], x[i]);
        float sum = __fadd_rn(__fadd_rn(__fadd_rn(x[0], x[1]), __fadd_rn(x[2], x[3])), __fadd_rn(__fadd_rn(x[4], x[5]), __fadd_rn(x[6], x[7])));
#pragma unroll
        for (int s = 1; s < D / 8; s <<= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, s));
        if ((lane & 3) == u) mean = sum;
    }
    return __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(mean, 1.f / D), eps)));
}

// A row's codes and parameters to its tile (`tile` null: nowhere).
template <int D, bool IS_V>
__device__ __forceinline__ void store_codes(const float (&x)[8], uint8_t* tile, int in_tile, int lane, int l) {
    float lo = x[0], hi = x[0];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]);
        odd |= !(fabsf(x[i]) <= 3.402823466e38f);  // NaN or infinity
    }
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, s));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, s));
    }
    odd = __ballot_sync(0xffffffffu, odd) & (0xffu << (lane & 24));
    uint32_t m_bits = __bfloat16_as_ushort(__float2bfloat16_rd(lo));
    const float m = bf_low(m_bits);
    const float span = fmaxf(__fmul_rn(__fsub_rn(hi, m), 1.f / 15.f), 0.f);
    uint32_t s_bits = __bfloat16_as_ushort(__float2bfloat16_ru(fminf(span, 65280.f)));
    if (odd) m_bits = 0x7fc0u, s_bits = 0;
    const float step = bf_low(s_bits), inverse = step >= 0x1p-100f ? __frcp_rn(step) : 0.f;
    float c[8];
    bool edge = inverse == 0.f;  // some quotient is close to the middle between two codes, or the step is tiny
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = __fmul_rn(__fsub_rn(x[i], m), inverse);
        c[i] = rintf(q), edge |= fabsf(q - c[i]) > 0.5f - 0x1p-16f;
    }
    if (edge) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = step > 0.f ? rintf(__fdiv_rn(__fsub_rn(x[i], m), step)) : 0.f;
    }
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= (uint32_t)fminf(fmaxf(c[i], 0.f), 15.f) << (4 * (IS_V ? i : k_place(i)));
    word = k_transpose(word, lane);
    if (IS_V) word = nibble_step(word, 4, 0x0000ffffu, lane);
    if (tile) {
        *reinterpret_cast<uint32_t*>(tile + in_tile * (D / 2) + word_at<D>(l, IS_V)) = word;
        if ((l & 7) == 0) *reinterpret_cast<uint32_t*>(tile + kKvqTile * D / 2 + in_tile * (D / 16) + (l >> 3) * 4) = s_bits | m_bits << 16;
    }
}

// The work is in groups of kSets sets of rows: a token's groups of query heads, then of K, then of V; a warp takes
// `per_warp` groups of one token.
template <int D, bool BF>
__global__ void __launch_bounds__(kThreads, 5) kvq_append_kernel(const KvqView v, const KvqRows q, const KvqRows k, const KvqRows val,
                                                              const KvqRows q_out, const Transform tr, const int q_heads,
                                                              const int q_groups, const int kv_groups, const int per_warp) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kStep = kSets * kRows;  // lanes of a row, rows of a warp, heads of a group
    constexpr int kTileBytes = kKvqTile * kvq_token_bytes(D);
    grid_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const int groups = q_groups + 2 * kv_groups, shares = (groups + per_warp - 1) / per_warp;
    const int64_t all = (int64_t)v.num_tokens * shares, step_of_grid = (int64_t)gridDim.x * kWarps;

    for (int64_t share = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); share < all; share += step_of_grid) {
        const int token = (int)(share / shares), first = (int)(share - (int64_t)token * shares) * per_warp;
        const int last = min(groups, first + per_warp);
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
        load(first, raw);

        const Slot slot = find_slot(v, token, kTileBytes);
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
        uint8_t* const tile0 = slot.stored ? v.base + slot.off : nullptr;
        const int in_tile = slot.pos & 15;

#pragma unroll 1
        for (int group = first; group < last; ++group) {
            uint4 now[kSets];
#pragma unroll
            for (int u = 0; u < kSets; ++u) now[u] = raw[u];
            if (group + 1 < last) load(group + 1, raw);
            if (group < q_groups) {
                const float scales = tr.q_norm ? row_scales<D, BF>(now, tr.eps, lane) : 0.f;
                const float4* weight = tr.q_norm ? reinterpret_cast<const float4*>(tr.q_norm + 8 * l) : nullptr;
                const int head0 = group * kStep + sub;
                uint16_t* p = q_out.data + token * q_out.s_token + head0 * q_out.s_head + 8 * l;
#pragma unroll
                for (int u = 0; u < kSets; ++u) {
                    float x[8];
                    unpack8<BF>(now[u], x);
                    turn_row(x, weight ? __shfl_sync(0xffffffffu, scales, (lane & ~3) | u) : 0.f, weight, turn);
                    if (head0 + u * kRows < q_heads) *reinterpret_cast<uint4*>(p + u * kRows * q_out.s_head) = pack8<BF>(x);
                }
            } else if (group < q_groups + kv_groups) {
                const float scales = tr.k_norm ? row_scales<D, BF>(now, tr.eps, lane) : 0.f;
                const float4* weight = tr.k_norm ? reinterpret_cast<const float4*>(tr.k_norm + 8 * l) : nullptr;
                const int head0 = (group - q_groups) * kStep + sub;
#pragma unroll 1
                for (int u = 0; u < kSets && head0 - sub + u * kRows < v.kv_heads; ++u) {
                    float x[8];
                    unpack8<BF>(u == 0 ? now[0] : u == 1 ? now[1] : u == 2 ? now[2] : now[3], x);
                    turn_row(x, weight ? __shfl_sync(0xffffffffu, scales, (lane & ~3) | u) : 0.f, weight, turn);
                    const int head = head0 + u * kRows;
                    store_codes<D, false>(x, tile0 && head < v.kv_heads ? tile0 + head * v.s_head : nullptr, in_tile, lane, l);
                }
            } else {
                const int head0 = (group - q_groups - kv_groups) * kStep + sub;
#pragma unroll 1
                for (int u = 0; u < kSets && head0 - sub + u * kRows < v.kv_heads; ++u) {
                    float x[8];
                    unpack8<BF>(u == 0 ? now[0] : u == 1 ? now[1] : u == 2 ? now[2] : now[3], x);
                    const int head = head0 + u * kRows;
                    store_codes<D, true>(x, tile0 && head < v.kv_heads ? tile0 + v.s_kv + head * v.s_head : nullptr, in_tile, lane, l);
                }
            }
        }
    }
}

template <int D, bool BF>
__global__ void __launch_bounds__(kThreads) kvq_read_kernel(const KvqView v, const KvqRows k, const KvqRows val, const int sets_per_token) {
    constexpr int kRowSets = kSets;
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    constexpr int kTileBytes = kKvqTile * kvq_token_bytes(D);
    grid_begin();
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int token = (int)(item / sets_per_token);
    if (token >= v.num_tokens) return;
    const int row0 = (int)(item - (int64_t)token * sets_per_token) * (kRows * kRowSets) + sub;
    const Slot slot = find_slot(v, token, kTileBytes);
    if (!slot.stored) {
        if (lane == 0) kvq_error(v, slot.known ? kErrBadBlock : kErrBadLength);
        return;
    }
    const int in_tile = slot.pos & 15;
    uint32_t word[kRowSets], par[kRowSets];
#pragma unroll
    for (int u = 0; u < kRowSets; ++u) {
        const int row = row0 + u * kRows;
        word[u] = par[u] = 0;
        if (row < 2 * v.kv_heads) {
            const bool is_v = row >= v.kv_heads;
            const uint8_t* tile = v.base + slot.off + (is_v ? row - v.kv_heads : row) * v.s_head + (is_v ? v.s_kv : 0);
            word[u] = *reinterpret_cast<const uint32_t*>(tile + in_tile * (D / 2) + word_at<D>(l, is_v));
            par[u] = *reinterpret_cast<const uint32_t*>(tile + kKvqTile * D / 2 + in_tile * (D / 16) + (l >> 3) * 4);
        }
    }
#pragma unroll
    for (int u = 0; u < kRowSets; ++u) {
        const int row = row0 + u * kRows;
        const bool is_v = row >= v.kv_heads;
        const uint32_t of_k = k_transpose(word[u], lane), of_v = nibble_step(of_k, 4, 0x0000ffffu, lane);
        const uint32_t w = is_v ? of_v : of_k;
        const float s = bf_low(par[u]), m = bf_high(par[u]);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = __fadd_rn(__fmul_rn((float)((w >> (4 * (is_v ? i : k_place(i)))) & 15), s), m);
            if (!BF && fabsf(x[i]) > 65504.f) x[i] = copysignf(65504.f, x[i]);  // the span's ends were rounded outwards
        }
        const KvqRows& out = is_v ? val : k;
        if (row < 2 * v.kv_heads && out.data)
            *reinterpret_cast<uint4*>(out.data + token * out.s_token + (is_v ? row - v.kv_heads : row) * out.s_head + 8 * l) =
                pack8<BF>(x);
    }
}

}  // namespace

remp_status kvq_view(const remp_kvq_pool* pool, const remp_kvq_batch* batch, KvqView* v) {
    if (!pool || !batch) return fail(REMP_ERR_INVALID_ARG, "null pool or batch");
    const int64_t tb = remp_kvq_token_bytes(pool->head_dim);
    if (tb < 0) return (remp_status)tb;
    if (pool->block_size < kKvqTile || pool->block_size % kKvqTile)
        return fail(REMP_ERR_SHAPE, "block_size must be a multiple of 16");
    if (pool->kv_heads < 1) return fail(REMP_ERR_SHAPE, "kv_heads must be positive");
    if (pool->layer < 0) return fail(REMP_ERR_INVALID_ARG, "negative layer");
    if (pool->shard.stride_token && pool->shard.stride_token != tb)
        return fail(REMP_ERR_SHAPE, "token rows of a 4-bit cache are dense");
    const remp_model_shape m = {1, pool->kv_heads, (int32_t)tb, pool->block_size, 1};
    TopoMap T;
    T.heads_per_rank = pool->kv_heads;
    ShardView s;
    if (remp_status st = resolve_shard(pool->shard, T, 1, m, &s)) return st;
    if (s.s_head < pool->block_size * tb) return fail(REMP_ERR_SHAPE, "stride_head must hold a head slice");
    if (s.nb > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "block ids are 32-bit");
    const remp_block_tables& bt = batch->tables;
    if (bt.num_seqs < 0 || bt.max_blocks_per_seq < 0 || batch->num_tokens < 0 || batch->max_queries < 0)
        return fail(REMP_ERR_INVALID_ARG, "negative batch dimensions");
    if (bt.num_seqs > kKvqMost || batch->num_tokens > kKvqMost) return fail(REMP_ERR_SHAPE, "too many sequences or tokens");
    if (batch->num_tokens > 0 && (!bt.seq_lens || !batch->query_start || (bt.max_blocks_per_seq > 0 && !bt.block_tables)))
        return fail(REMP_ERR_INVALID_ARG, "null seq_lens, block_tables or query_start");
    v->base = reinterpret_cast<uint8_t*>(s.base + (uint64_t)((int64_t)pool->layer * s.s_layer));
    v->s_kv = s.s_kv, v->s_block = s.s_block, v->s_head = s.s_head;
    v->nb = (int32_t)s.nb, v->kv_heads = pool->kv_heads, v->block_tiles = pool->block_size / kKvqTile;
    v->max_blocks = bt.max_blocks_per_seq, v->num_seqs = bt.num_seqs, v->num_tokens = bt.num_seqs ? batch->num_tokens : 0;
    v->seq_lens = bt.seq_lens, v->tables = bt.block_tables, v->query_start = batch->query_start;
    v->error = batch->error;
    return REMP_OK;
}

remp_status kvq_rows(const remp_kvq_rows* r, int32_t tokens, int32_t heads, int32_t head_dim, bool written, const char* name, KvqRows* out) {
    if (!r || !r->data) return fail(REMP_ERR_INVALID_ARG, std::string("null ") + name);
    const int64_t s_token = tokens > 1 ? r->stride_token : 0, s_head = heads > 1 ? r->stride_head : 0;
    if ((reinterpret_cast<uint64_t>(r->data) & 15) || (s_token & 7) || (s_head & 7))
        return fail(REMP_ERR_SHAPE, std::string(name) + ": base must be 16-byte aligned and strides multiples of 8 elements");
    const auto apart = [&](int64_t stride) { return stride >= head_dim || stride <= -head_dim; };
    if (heads > 1 && !apart(s_head) && (written || s_head != 0)) return fail(REMP_ERR_SHAPE, std::string(name) + ": heads overlap");
    if (tokens > 1 && !apart(s_token) && written) return fail(REMP_ERR_SHAPE, std::string(name) + ": tokens overlap");
    out->data = static_cast<uint16_t*>(r->data);
    out->s_token = s_token, out->s_head = s_head;
    return REMP_OK;
}

static remp_status check_dtype(int32_t dtype) {
    return dtype == REMP_DTYPE_BFLOAT || dtype == REMP_DTYPE_HALF ? REMP_OK : fail(REMP_ERR_INVALID_ARG, "unknown dtype");
}

}  // namespace remp

using namespace remp;

extern "C" int64_t remp_kvq_token_bytes(int32_t head_dim) {
    if (head_dim != 64 && head_dim != 128 && head_dim != 256)
        return fail(REMP_ERR_SHAPE, "head_dim of a 4-bit cache must be 64, 128 or 256");
    return kvq_token_bytes(head_dim);
}

extern "C" remp_status remp_kvq_append(const remp_kvq_pool* pool, const remp_kvq_batch* batch, const remp_kvq_rows* q,
                                       const remp_kvq_rows* k, const remp_kvq_rows* v, const remp_kvq_rows* q_out,
                                       int32_t q_heads, int32_t dtype, const remp_kvq_transform* transform,
                                       void* stream_) {
    KvqView view;
    KvqRows rq{nullptr, 0, 0}, rk, rv, ro{nullptr, 0, 0};
    if (remp_status st = kvq_view(pool, batch, &view)) return st;
    if (remp_status st = check_dtype(dtype)) return st;
    const int32_t d = pool->head_dim;
    if (q_heads < 0 || (q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr))
        return fail(REMP_ERR_INVALID_ARG, "q, q_out and q_heads go together");
    Transform tr{nullptr, nullptr, nullptr, nullptr, 0.f, 0, 0, 0};
    if (transform) {
        tr = Transform{transform->q_norm, transform->k_norm, transform->rope, transform->positions, transform->eps,
                       transform->rope_rows, transform->rotary_dim, transform->interleaved};
        if ((reinterpret_cast<uint64_t>(tr.q_norm) | reinterpret_cast<uint64_t>(tr.k_norm) | reinterpret_cast<uint64_t>(tr.rope)) & 15)
            return fail(REMP_ERR_SHAPE, "norm weights and the rotation table must be 16-byte aligned");
        if (!(tr.eps >= 0.f)) return fail(REMP_ERR_INVALID_ARG, "eps must not be negative");
        if (tr.rope && (tr.rotary_dim < 16 || tr.rotary_dim % 16 || tr.rotary_dim > d || tr.rope_rows < 0))
            return fail(REMP_ERR_SHAPE, "rotary_dim must be a multiple of 16 and at most head_dim");
        if (!tr.rope) tr.rotary_dim = 0;
    }
    if (view.num_tokens == 0) return REMP_OK;
    if (q_heads) {
        if (remp_status st = kvq_rows(q, view.num_tokens, q_heads, d, false, "q", &rq)) return st;
        if (remp_status st = kvq_rows(q_out, view.num_tokens, q_heads, d, true, "q_out", &ro)) return st;
    }
    if (remp_status st = kvq_rows(k, view.num_tokens, pool->kv_heads, d, false, "k", &rk)) return st;
    if (remp_status st = kvq_rows(v, view.num_tokens, pool->kv_heads, d, false, "v", &rv)) return st;
    const int64_t rows = (int64_t)q_heads + 2 * (int64_t)pool->kv_heads;
    const int heads = 32 / (d / 8) * kSets;  // of a group
    if (rows > 0x7fffffffLL - 3 * heads) return fail(REMP_ERR_SHAPE, "too many heads");
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    const int q_groups = (q_heads + heads - 1) / heads, kv_groups = (pool->kv_heads + heads - 1) / heads, groups = q_groups + 2 * kv_groups;
    // a token to a warp when that fills the GPU, else a group
    const int per_warp = view.num_tokens >= sms * 20 ? groups : 1;
    const int64_t shares = (int64_t)view.num_tokens * ((groups + per_warp - 1) / per_warp);
    const int64_t grid = std::min<int64_t>((shares + kWarps - 1) / kWarps, (int64_t)sms * 40);
    const bool bf = dtype == REMP_DTYPE_BFLOAT;
    const auto kernel = d == 64    ? (bf ? kvq_append_kernel<64, true> : kvq_append_kernel<64, false>)
                        : d == 128 ? (bf ? kvq_append_kernel<128, true> : kvq_append_kernel<128, false>)
                                   : (bf ? kvq_append_kernel<256, true> : kvq_append_kernel<256, false>);
    REMP_CUDA(launch_after(kernel, grid, kThreads, 0, static_cast<cudaStream_t>(stream_), view, rq, rk, rv, ro, tr, (int)q_heads, q_groups, kv_groups,
                           per_warp));
    return REMP_OK;
}

extern "C" remp_status remp_kvq_read(const remp_kvq_pool* pool, const remp_kvq_batch* batch, const remp_kvq_rows* k_out,
                                     const remp_kvq_rows* v_out, int32_t dtype, void* stream_) {
    KvqView view;
    KvqRows rk{nullptr, 0, 0}, rv{nullptr, 0, 0};
    if (remp_status st = kvq_view(pool, batch, &view)) return st;
    if (remp_status st = check_dtype(dtype)) return st;
    const int32_t d = pool->head_dim;
    if (view.num_tokens == 0 || (!k_out && !v_out)) return REMP_OK;
    if (k_out)
        if (remp_status st = kvq_rows(k_out, view.num_tokens, pool->kv_heads, d, true, "k_out", &rk)) return st;
    if (v_out)
        if (remp_status st = kvq_rows(v_out, view.num_tokens, pool->kv_heads, d, true, "v_out", &rv)) return st;
    const int per_item = 32 / (d / 8) * kSets;
    const int64_t sets = (2 * (int64_t)pool->kv_heads + per_item - 1) / per_item;
    const int64_t grid = (view.num_tokens * sets + kWarps - 1) / kWarps;
    if (grid > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "too many rows for one call");
    const bool bf = dtype == REMP_DTYPE_BFLOAT;
    const auto kernel = d == 64    ? (bf ? kvq_read_kernel<64, true> : kvq_read_kernel<64, false>)
                        : d == 128 ? (bf ? kvq_read_kernel<128, true> : kvq_read_kernel<128, false>)
                                   : (bf ? kvq_read_kernel<256, true> : kvq_read_kernel<256, false>);
    REMP_CUDA(launch_after(kernel, grid, kThreads, 0, static_cast<cudaStream_t>(stream_), view, rk, rv, (int)sets));
    return REMP_OK;
}
