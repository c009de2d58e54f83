// The weight that attention gives to cached positions (rules: include/remp.h).
//
// Mathematics: weight of key j += sum over rows r that see it of 2^(q_r.k_j * scale - lse_r), with scale and lse in powers of
// two. The rows' sums are given, so every key is on its own: no parts, no merging, no atomics.
// Rounding: scores, probabilities and sums are in 32 bits; nothing is rounded to fewer.
//
// Bound: HBM for few rows (K is read once). A tile is 16 tokens of one head, held by a warp in operand registers for all
// rows: lane (g, t) loads 16 bytes of tokens g and g + 8 at dims 32i + 8t, which are the operands of two matrix instructions if the
// queries come in the same order of dims, so K needs no shared memory. Work is the list of all (sequence, KV head, tile), cut evenly
// over the warps of the grid; a warp asks for its next tile before it works on this one.

#include "remp_kv_boxes.h"
#include "remp_kv_weigh.h"
#include "remp_kvq_device.h"

namespace remp {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
// Which kernel: this one takes up to 24 rows of a sequence, and more where sequences and KV heads fill the GPU but are so short that a
// thread block for each costs more than it saves: this one takes a time for each tile and set of 8 rows (0.3 ns for the whole GPU,
// 0.6 with 256 dims), the wide one for each tile, whatever the rows up to 256 (1.0 to 1.3), and for each sequence and KV head about 30
// ns. Here and there, us in a graph, 8 KV heads of 128 dims: 24 rows, 300 sequences of 500 tokens 117 and 150, 64 of 500 33 and 41, 24
// of 3000 59 and 70, 2 of 16000 31 and 29; 32 rows 143 and 150, 37 and 41, 70 and 68, 35 and 29; 48 rows 188 and 156, 45 and 43, 90 and
// 70, 45 and 29; 1000 of 50 57, 68 and 86, and 266 to 291; 8 of 100, 64 rows 16 and 12. 256 dims, 32 rows: 244 and 170, 57 and 51.
bool wide_takes(int head_dim, int64_t rows, int64_t units, int sms, int64_t tokens) {
    const int64_t sets = (rows + 7) / 8, tiles = (tokens + kKvqTile - 1) / kKvqTile;
    return rows > 24 && (units <= sms || tiles * (2 * sets - 3) > (head_dim == 256 ? 100 : 200));
}

struct Seq {
    KvqSpan x;
    KvTiles tiles;
    int rows, steps;
};

__device__ __forceinline__ Seq seq_of(const WeighArgs& a, int s) {
    Seq r;
    r.x = kvq_span(a.v.query_start[s], a.v.query_start[s + 1], a.v.seq_lens[s], a.v.num_tokens, a.room);
    r.rows = r.x.queries * a.group;
    // fresh: every position is written
    r.tiles = a.fresh ? kv_tiles(r.x, 0, 0, 0) : kv_tiles(r.x, r.x.first_pos, a.window, a.first);
    r.steps = r.rows ? r.tiles.sinks + r.tiles.rest : 0;
    return r;
}

template <int D, bool BF>
__global__ void __launch_bounds__(kThreads, D == 256 ? 1 : 2) kv_weigh_kernel(const __grid_constant__ WeighArgs a) {
    __shared__ long long warp_sum[kWarps];
    __shared__ int first_at[kWarps], first_seq[kWarps];  // where a warp's share begins: sequences from here, at this place in the list
    constexpr int kChunks = D / 32;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const KvView& v = a.v;
    const int spt = (v.num_seqs + kThreads - 1) / kThreads;
    grid_begin();

    const int s0 = min(v.num_seqs, tid * spt), s1 = min(v.num_seqs, s0 + spt);
    long long mine = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const Seq q = seq_of(a, s);
        mine += (long long)q.steps * v.kv_heads;
        if (blockIdx.x == 0 && kvq_span_bad(q.x, v.seq_lens[s])) kvq_error(v, kErrBadLength);
    }
    long long before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += up;
    }
    if (lane == 31) warp_sum[wid] = before;
    __syncthreads();
    before -= mine;
    long long total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const long long x = warp_sum[w];
        if (w < wid) before += x;
        total += x;
    }
    if (total > 0x40000000) {  // 2^30 tiles, as for attention
        if (blockIdx.x == 0 && tid == 0) kvq_error(v, kErrOverflow);
        return;
    }
    // a warp's share of the list
    const long long warps = (long long)gridDim.x * kWarps, per = (total + warps - 1) / warps, block0 = (long long)blockIdx.x * kWarps * per;
    if (block0 >= total) return;
    if (mine > 0 && before < block0 + kWarps * per && before + mine > block0) {
        const long long from = max(0LL, (before - block0 + per - 1) / per);
#pragma unroll 1
        for (long long w = from; w < kWarps && block0 + w * per < before + mine; ++w) first_seq[w] = s0, first_at[w] = (int)min(block0 + w * per - before, 0x7fffffffLL);
    }
    __syncthreads();
    const long long w0 = block0 + wid * per;
    const int todo = (int)min(per, total - w0);
    if (todo <= 0) return;

    Seq q{};
    int seq = first_seq[wid], head = 0, step = 0, left_in = first_at[wid];  // places before the share's first in its thread's sequences
    uint32_t k[kChunks][2][4], next[kChunks][2][4];
    int key0 = 0, next_key = 0;
    bool there = false, next_there = false;
    // Moves to the list's next place and asks for its tile.
    const auto advance = [&](bool begin) {
        if (begin) {
#pragma unroll 1
            for (;; ++seq) {
                q = seq_of(a, seq);
                const long long n = (long long)q.steps * v.kv_heads;
                if (left_in < n) break;
                left_in -= (int)n;
            }
            head = left_in / q.steps, step = left_in - head * q.steps;
        } else if (++step == q.steps) {
            step = 0;
            if (++head == v.kv_heads) {
                head = 0;
#pragma unroll 1
                do q = seq_of(a, ++seq);
                while (q.steps == 0);
            }
        }
        const int tile = step < q.tiles.sinks ? step : q.tiles.tile0 + step - q.tiles.sinks;
        next_key = tile * kKvqTile;
        // tiles that no row sees are in the list of a fresh call only, to get 0; their pages may have been given back
        const bool seen = next_key + kKvqTile > kvq_first_key(q.x.first_pos, a.window) || next_key < a.first;
        const int in_row = tile / v.block_tiles, id = seen ? __ldg(v.tables + (int64_t)seq * v.max_blocks + in_row) : -1;
        next_there = (uint32_t)id < (uint32_t)v.nb;
        if (seen && !next_there && lane == 0) kvq_error(v, kErrBadBlock);
        const uint8_t* src = v.base + (int64_t)id * v.s_block + (int64_t)head * v.s_head + (int64_t)(tile - in_row * v.block_tiles) * kKvqTile * v.s_token + g * v.s_token + 16 * t;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (next_there && next_key + g + 8 * h < q.x.len) x = __ldcs(reinterpret_cast<const uint4*>(src + 8 * h * v.s_token + 64 * c));
                next[c][h][0] = x.x, next[c][h][1] = x.y, next[c][h][2] = x.z, next[c][h][3] = x.w;
            }
    };
    advance(true);
#pragma unroll 1
    for (int i = 0; i < todo; ++i) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int x = 0; x < 4; ++x) k[c][h][x] = next[c][h][x];
        key0 = next_key, there = next_there;
        const Seq w = q;
        const int w_head = head;
        float* const to = a.weights + ((int64_t)seq * v.kv_heads + head) * a.stride + key0;
        if (i + 1 < todo) advance(false);
        float sum[2] = {0.f, 0.f};
        const int high = w.x.first_pos + w.x.queries - 1;
        if (there && key0 <= high) {
#pragma unroll 1
            for (int r0 = 0; r0 < w.rows; r0 += 8) {
                // rows before the tile see nothing of it; the last one of these rows is the farthest
                if (w.x.first_pos + kv_token_of(a.by_group, min(r0 + 7, w.rows - 1)) < key0) continue;
                const int r = r0 + g, row = min(r, w.rows - 1), token = kv_token_of(a.by_group, row);
                const uint16_t* src = a.q.data + (int64_t)(w.x.q0 + token) * a.q.s_token + (int64_t)(w_head * a.group + row - token * a.group) * a.q.s_head + 8 * t;
                uint4 b[kChunks];
#pragma unroll
                for (int c = 0; c < kChunks; ++c) b[c] = __ldg(reinterpret_cast<const uint4*>(src + 32 * c));
                float norm[2];
                int limit[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int rr = r0 + 2 * t + e, one = min(rr, w.rows - 1), at = kv_token_of(a.by_group, one);
                    const float l = __ldg(a.lse + (int64_t)(w.x.q0 + at) * a.q_heads + w_head * a.group + one - at * a.group);
                    norm[e] = rr < w.rows && l != -INFINITY ? l * 1.4426950408889634f : INFINITY;
                    limit[e] = w.x.first_pos + at;
                }
                float even[4] = {0.f, 0.f, 0.f, 0.f}, odd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const uint32_t x[4] = {k[c][0][0], k[c][1][0], k[c][0][1], k[c][1][1]}, y[4] = {k[c][0][2], k[c][1][2], k[c][0][3], k[c][1][3]};
                    mma_rows<BF>(even, x, b[c].x, b[c].y);
                    mma_rows<BF>(odd, y, b[c].z, b[c].w);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float p = exp2_approx(fmaf(even[2 * h + e] + odd[2 * h + e], a.scale_log2, -norm[e]));
                        if (norm[e] != INFINITY && kv_sees(limit[e], key0 + g + 8 * h, a.window, a.first)) sum[h] += p;
                    }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
        }
        if (t < 2) {
            const int key = key0 + g + 8 * t;
            if (key < w.x.len) {
                const float x = t ? sum[1] : sum[0];
                float* p = to + g + 8 * t;
                *p = a.fresh || key >= w.x.first_pos ? x : *p + x;
            }
        }
    }
}

}  // namespace

}  // namespace remp

using namespace remp;

extern "C" remp_status remp_kv_weigh(const remp_kv_pool* pool, const remp_kvq_batch* batch, const remp_kvq_rows* q, int32_t q_heads,
                                     int32_t dtype, float scale, int32_t window, int32_t first, const float* lse, float* weights,
                                     int64_t stride, int32_t fresh, void* stream_) {
    WeighArgs a{};
    if (remp_status st = kv_view(pool, batch, &a.v)) return st;
    if (remp_status st = kvq_dtype(dtype)) return st;
    if (remp_status st = kv_mask(scale, window, first)) return st;
    if (remp_status st = kv_group(q_heads, pool->kv_heads, batch->num_tokens, &a.group, &a.by_group)) return st;
    if (stride < 0) return fail(REMP_ERR_INVALID_ARG, "negative stride of the weights");
    if (a.v.num_tokens == 0) return REMP_OK;
    if (!lse || (stride > 0 && !weights)) return fail(REMP_ERR_INVALID_ARG, "null lse or weights");
    if (remp_status st = kvq_rows(q, a.v.num_tokens, q_heads, pool->head_dim, false, "q", &a.q)) return st;
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    a.lse = lse, a.weights = weights, a.stride = stride;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.q_heads = q_heads, a.window = window, a.first = window > 0 ? first : 0, a.fresh = fresh != 0;
    a.room = (int32_t)std::min<int64_t>(std::min<int64_t>((int64_t)a.v.max_blocks * a.v.block_tiles * kKvqTile, kKvqMost), stride);
    const bool bf = dtype == REMP_DTYPE_BFLOAT;
    const int d = pool->head_dim;
    const int64_t seen = window > 0 && !fresh ? std::min<int64_t>(a.room, (int64_t)window + a.first + batch->max_queries) : a.room;
    if (wide_takes(d, (int64_t)std::min(batch->max_queries, batch->num_tokens) * a.group, (int64_t)a.v.num_seqs * pool->kv_heads, sms, seen) && kv_boxes_take(a.v)) {
        REMP_CUDA(launch_kv_weigh_wide(a, d, bf, sms, static_cast<cudaStream_t>(stream_)));
        return REMP_OK;
    }
    const auto kernel = d == 64    ? (bf ? kv_weigh_kernel<64, true> : kv_weigh_kernel<64, false>)
                        : d == 128 ? (bf ? kv_weigh_kernel<128, true> : kv_weigh_kernel<128, false>)
                                   : (bf ? kv_weigh_kernel<256, true> : kv_weigh_kernel<256, false>);
    REMP_CUDA(launch_after(kernel, d == 256 ? sms : 2 * sms, kThreads, 0, static_cast<cudaStream_t>(stream_), a));
    return REMP_OK;
}
