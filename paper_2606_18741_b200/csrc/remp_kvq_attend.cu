// Attention over the 4-bit cache for few queries per sequence (decode, drafts, short continuations).
//
// Mathematics. With a key's codes c, step s and minimum m for each group of 64 dims, q.k = sum over groups of
// s*(q.c) + m*sum(q); with a value's, sum p*v = sum (p*s)*(c - 8) + sum p*(m + 8s). So the matrix instructions work on
// bare codes: a key's code in the low bits of a half is the subnormal c*2^-24, exact, and taking codes out of a word is an
// AND (and a shift for half of them); codes left at bits 4..7 count 16-fold, which the query's other half of the dims (K) or
// the output row (V) undoes. The factor 2^-24 leaves with the scale. A value's codes take one subtraction more.
// Softmax with a running reference: p = 2^(x - ref), and p times the largest step seen stays at or below 2^15. A
// reference moves only when a score (or a step) passes that bound, by kSlack further than needed, which one vote for each
// 32 tokens finds out; accumulators are seldom rescaled, and p*s keeps 11 bits over 29 powers of two.
// Rounding: q is exact in half after a power of two per row; p*s is rounded to half (kvq_values); scores, references, sums of p, sums of p*m and outputs are in 32 bits.
//
// Roles: a tile is 16 tokens of one head. S^T[16 tokens][8 rows] = K.Q^T and O^T[D][8 rows] += V^T.P^T, so the eight query
// heads of a KV head fill the 8 columns of m16n8k16; P^T goes from accumulator to operand layout with one
// matrix transpose for each 8 tokens. NT = 2 takes 16 rows and is used when 8 do not hold a sequence's rows.
//
// Bound: HBM. Work is the list of all (sequence, row block, KV head, step of two tiles), cut evenly over the thread blocks
// and within one evenly over its warps, so ragged batches and single long sequences fill the GPU alike. A warp streams
// its steps through two buffers in shared memory with 16-byte asynchronous copies and needs no block-wide
// barrier until its share is done. Parts of a sequence are merged in the block, and across blocks by the block that
// arrives last (a counter; nobody waits), always in the order of the list: the result does not depend on timing.

#include "remp_kvq_device.h"

namespace remp {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr float kNoRef = -1e30f;  // reference of a row that has seen nothing; finite, so that -inf - kNoRef is -inf
constexpr float kSlack = 4.f;     // log2: a new reference leaves room for scores up to 4 higher and steps up to 16 times larger
constexpr float kTopStep = 1.f / 1024;  // steps below this are not looked at
constexpr int kStepTiles = 2, kStepTokens = kStepTiles * kKvqTile;

struct AttendArgs {
    KvqView v;
    KvqRows q, out;
    float* lse;
    uint8_t* workspace;
    float scale_log2;  // softmax scale * log2(e)
    int32_t group, q_heads, window, bf;
    int32_t spt;       // sequences of one thread of the block-wide scan
};

struct Seq {  // one sequence's share of the list
    int len, q0, rows;      // cached tokens, first row of the batch, query rows (queries * group)
    int tile0, tiles;       // tiles that its rows see
    int steps;              // of kStepTiles; at least one, so that rows which see nothing are written too
    int first_pos;          // position of its first query
    int blocks;             // row blocks
};

template <int RB>
__device__ __forceinline__ Seq seq_of(const AttendArgs& a, int s) {
    Seq r;
    const int qs = max(0, a.v.query_start[s]), qe = min(a.v.num_tokens, a.v.query_start[s + 1]);
    const int n = max(0, qe - qs);
    const int64_t room = (int64_t)a.v.max_blocks * a.v.block_tiles * kKvqTile;
    const int len = a.v.seq_lens[s];
    r.len = (int)min((int64_t)max(len, 0), room);
    r.q0 = qs, r.rows = n * a.group, r.blocks = (r.rows + RB - 1) / RB;
    r.first_pos = len - n;
    const int from = a.window > 0 ? max(0, r.first_pos - a.window + 1) : 0;
    r.tile0 = min(from, r.len) / kKvqTile;
    r.tiles = (r.len + kKvqTile - 1) / kKvqTile - r.tile0;
    r.steps = max(1, (r.tiles + kStepTiles - 1) / kStepTiles);
    return r;
}

template <int RB>
__device__ __forceinline__ long long steps_of(const AttendArgs& a, int s) {
    const Seq q = seq_of<RB>(a, s);
    return (long long)q.blocks * a.v.kv_heads * q.steps;
}

struct Cursor {  // a place in the list
    Seq q;
    int s, head, block, step;  // sequence, KV head, row block, step
};

template <int RB>
__device__ __forceinline__ void next_unit(const AttendArgs& a, Cursor& c) {
    c.step = 0;
    if (++c.block < c.q.blocks) return;
    c.block = 0;
    if (++c.head < a.v.kv_heads) return;
    c.head = 0;
    do {
        if (++c.s >= a.v.num_seqs) return;
        c.q = seq_of<RB>(a, c.s);
    } while (c.q.rows == 0);
}

struct Part {  // what a warp leaves of a unit that it did not see whole
    long long from, to;  // the unit's steps in the list
    int q0, row0, rows, head;
    int live;
};

template <int D, int NT>
struct Sizes {
    static constexpr int kRows = 8 * NT;
    static constexpr int kTileBytes = kKvqTile * kvq_token_bytes(D);
    static constexpr int kStage = 2 * kTileBytes;                    // K and V of a tile
    static constexpr int kBuffer = kStepTiles * kStage;
    static constexpr int kPitch = D + 4;                             // floats of a part's row: spreads the banks
    static constexpr int kPart = kRows * (kPitch + 2) * 4;           // rows, references, sums
    static constexpr int kRing = 2 * kBuffer > kPart ? 2 * kBuffer : kPart;  // the tail part reuses the buffers
    static constexpr int kWarpBytes = (kRing + kPart + 127) / 128 * 128;
    static constexpr int kBytes = kWarps * kWarpBytes;
    static constexpr int kSlotFloats = kRows * (D + 2);  // a part in the workspace
};

// out[row][4 dims] = x
__device__ __forceinline__ void store4(const AttendArgs& a, const Part& p, int r, int d, const float4& x) {
    const int row = p.row0 + r, token = p.q0 + row / a.group, head = p.head * a.group + row % a.group;
    uint2 w;
    if (a.bf) {
        const __nv_bfloat162 u = __floats2bfloat162_rn(x.x, x.y), v = __floats2bfloat162_rn(x.z, x.w);
        w = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
    } else {
        const __half2 u = __floats2half2_rn(x.x, x.y), v = __floats2half2_rn(x.z, x.w);
        w = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
    }
    *reinterpret_cast<uint2*>(a.out.data + token * a.out.s_token + head * a.out.s_head + d) = w;
}

__device__ __forceinline__ void store_lse(const AttendArgs& a, const Part& p, int r, float ref, float sum) {
    const int row = p.row0 + r;
    a.lse[(int64_t)(p.q0 + row / a.group) * a.q_heads + p.head * a.group + row % a.group] =
        sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
}

// Merge `n` parts (n >= 1; part i's rows at rows(i), references at refs(i), sums behind them) into the output or, with
// `slot`, into a part of the workspace. The whole thread block works on it.
template <int D, int NT, class Rows>
__device__ __forceinline__ void merge(const AttendArgs& a, const Part& p, int n, int pitch, const Rows& part, float* slot) {
    constexpr int R = 8 * NT;
    for (int e = threadIdx.x; e < p.rows * (D / 4); e += kThreads) {
        const int r = e / (D / 4), d = e % (D / 4) * 4;
        float ref = kNoRef;
        for (int i = 0; i < n; ++i) ref = fmaxf(ref, part(i)[R * pitch + r]);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
        for (int i = 0; i < n; ++i) {
            const float* x = part(i);
            const float w = exp2f(x[R * pitch + r] - ref);
            const float4 o = *reinterpret_cast<const float4*>(x + r * pitch + d);
            acc.x += w * o.x, acc.y += w * o.y, acc.z += w * o.z, acc.w += w * o.w;
            sum += w * x[R * pitch + R + r];
        }
        if (slot) {
            *reinterpret_cast<float4*>(slot + r * D + d) = acc;
            if (d == 0) slot[R * D + r] = ref, slot[R * D + R + r] = sum;
        } else {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            store4(a, p, r, d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
            if (d == 0 && a.lse) store_lse(a, p, r, ref, sum);
        }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, (D == 256 || NT == 2) ? 1 : 2) kvq_attend_kernel(const AttendArgs a) {
    using Z = Sizes<D, NT>;
    constexpr int RB = Z::kRows, G = D / kKvqGroup;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long scan[kThreads + 1];
    __shared__ long long warp_sum[kWarps];
    __shared__ Part parts[kWarps][2];
    __shared__ int last_of[2];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const KvqView& v = a.v;

    // ---- the list: steps before each thread's sequences ----
    {
        long long mine = 0;
        const int s0 = min(v.num_seqs, tid * a.spt), s1 = min(v.num_seqs, s0 + a.spt);
        for (int s = s0; s < s1; ++s) {
            mine += steps_of<RB>(a, s);
            if (blockIdx.x == 0) {
                const int len = v.seq_lens[s];
                if (len < 0 || len > (int64_t)v.max_blocks * v.block_tiles * kKvqTile) kvq_error(v, kErrBadLength);
            }
        }
        long long incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        if (lane == 31) warp_sum[wid] = incl;
        if (tid < kWarps * 2) parts[tid >> 1][tid & 1].live = 0;
        __syncthreads();
        long long before = 0;
        for (int w = 0; w < wid; ++w) before += warp_sum[w];
        scan[tid + 1] = before + incl;
        if (tid == 0) scan[0] = 0;
        __syncthreads();
    }
    const long long total = scan[kThreads];
    const long long per = max((long long)kWarps, (total + gridDim.x - 1) / gridDim.x);
    const long long cta0 = blockIdx.x * per, cta1 = min(total, cta0 + per);
    if (cta0 >= total) return;
    const long long wper = (cta1 - cta0 + kWarps - 1) / kWarps;
    const long long w0 = min(cta1, cta0 + wid * wper), w1 = min(cta1, w0 + wper);

    uint8_t* ring = smem + wid * Z::kWarpBytes;
    float* head_part = reinterpret_cast<float*>(ring + Z::kRing);
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);

    if (w0 < w1) {
        // ---- the warp's first place ----
        Cursor c;  // of the loads, ahead of the work
        long long unit0;  // list index of step 0 of the unit at work
        {
            int lo = 0, hi = kThreads - 1;  // last thread whose sequences begin at or before w0
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (scan[mid] <= w0) lo = mid; else hi = mid - 1;
            }
            long long at = scan[lo];
            c.s = lo * a.spt;
            for (;; ++c.s) {
                c.q = seq_of<RB>(a, c.s);
                const long long n = (long long)c.q.blocks * v.kv_heads * c.q.steps;
                if (at + n > w0) break;
                at += n;
            }
            const long long in = w0 - at;
            const int unit = (int)(in / c.q.steps);
            c.step = (int)(in % c.q.steps), c.head = unit / c.q.blocks, c.block = unit - c.head * c.q.blocks;
            unit0 = w0 - c.step;
        }
        Cursor w = c;

        // ---- loads: ids of 32 blocks at a time in the lanes, blocks walked without a division ----
        int ids = -1, ids_seq = -1, ids_first = 0;
        int in_row = 0, in_block = 0;  // place of the next tile in its row of the table
        uint32_t absent = 0;           // tiles of either buffer that are not there
        const auto enter = [&]() {
            const int tile = c.q.tile0 + c.step * kStepTiles;
            in_row = tile / v.block_tiles, in_block = tile - in_row * v.block_tiles;
        };
        enter();
        const auto issue = [&](int buffer) {
            const uint8_t* base = v.base + (int64_t)c.head * v.s_head;
#pragma unroll
            for (int j = 0; j < kStepTiles; ++j) {
                bool there = c.step * kStepTiles + j < c.q.tiles;
                if (there) {
                    if (c.s != ids_seq || in_row < ids_first || in_row >= ids_first + 32) {
                        ids_seq = c.s, ids_first = in_row;
                        ids = in_row + lane < v.max_blocks ? v.tables[(int64_t)c.s * v.max_blocks + in_row + lane] : -1;
                    }
                    const int id = __shfl_sync(0xffffffffu, ids, in_row - ids_first);
                    there = (uint32_t)id < (uint32_t)v.nb;
                    if (there)
                        kvq_fetch_tile<D>(base + (int64_t)id * v.s_block + in_block * Z::kTileBytes, v.s_kv,
                                          ring_at + buffer * Z::kBuffer + j * Z::kStage, lane);
                    else if (lane == 0)
                        kvq_error(v, kErrBadBlock);
                    if (++in_block == v.block_tiles) in_block = 0, ++in_row;
                }
                const uint32_t bit = 1u << (buffer * kStepTiles + j);
                absent = there ? absent & ~bit : absent | bit;
            }
            if (++c.step == c.q.steps) {
                next_unit<RB>(a, c);
                enter();
            }
        };
        long long ahead = w0 + 1;
        issue(0);
        cp_async_commit();

        // ---- work ----
        int buffer = 0;
        for (long long x = w0; x < w1;) {
            const int head = w.head, row0 = w.block * RB;
            const int rows = min(RB, w.q.rows - row0);
            const long long unit1 = unit0 + w.q.steps, stop = min(unit1, w1);

            // queries of this lane's column g (+8): halves of the operand, their sums, and the exponent that was taken out
            uint32_t qf[NT][D / 16][2];
            float qsum[NT][G][2], back[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = row0 + min(8 * n + g, rows - 1);
                const bool real = 8 * n + g < rows;
                const uint16_t* src = a.q.data + (int64_t)(w.q.q0 + r / a.group) * a.q.s_token +
                                      (int64_t)(head * a.group + r % a.group) * a.q.s_head + 2 * t;
                kvq_load_queries<D>(src, a.bf != 0, real, t, qf[n], qsum[n], back[n], a.scale_log2);
            }
            // the positions of the first and the last row
            const int low_limit = w.q.first_pos + row0 / a.group, high_limit = w.q.first_pos + (row0 + rows - 1) / a.group;
            float o[NT][D / 16][4], ref[NT][2], sum[NT][2], low[NT][G][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
                ref[n][0] = ref[n][1] = kNoRef, sum[n][0] = sum[n][1] = 0.f;
#pragma unroll
                for (int i = 0; i < G; ++i) low[n][i][0] = low[n][i][1] = 0.f;
            }
            float top_step = kTopStep, room = 25.f;  // p * top_step <= 2^15: p <= 2^room

            for (; x < stop; ++x) {
                cp_async_wait<0>();
                __syncwarp();
                const uint8_t* buf = ring + buffer * Z::kBuffer;
                const uint32_t missing = absent >> (buffer * kStepTiles) & ((1u << kStepTiles) - 1);
                buffer ^= 1;
                if (ahead < w1) issue(buffer), ++ahead;
                cp_async_commit();
                const int key0 = (w.q.tile0 + w.step * kStepTiles) * kKvqTile;
                ++w.step;

                float s[kStepTiles][NT][4];
                uint32_t par[kStepTiles][2][G];
#pragma unroll
                for (int j = 0; j < kStepTiles; ++j) {
                    kvq_scores<D, NT>(buf + j * Z::kStage, g, t, qf, qsum, s[j]);
                    kvq_params<D>(buf + j * Z::kStage + Z::kTileBytes, g, par[j]);
                }
                if (missing || key0 + kStepTokens - 1 > low_limit || key0 + kStepTokens > w.q.len ||
                    (a.window > 0 && key0 <= high_limit - a.window)) {
                    // what a row does not see gets -infinity; the steps and minima of tokens that are not there, 0
#pragma unroll
                    for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int key = key0 + j * kKvqTile + g + 8 * h;
                            const bool there = key < w.q.len && !(missing >> j & 1);
#pragma unroll
                            for (int i = 0; i < G; ++i)
                                if (!there) par[j][h][i] = 0;
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int col = min(8 * n + 2 * t + e, rows - 1);
                                    const int limit = w.q.first_pos + (row0 + col) / a.group;
                                    if (!there || key > limit || (a.window > 0 && key <= limit - a.window))
                                        s[j][n][2 * h + e] = -INFINITY;
                                }
                        }
                }
                float over = -INFINITY, step = 0.f;
#pragma unroll
                for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < G; ++i) step = fmaxf(step, bf_low(par[j][h][i]));
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) over = fmaxf(over, fmaf(s[j][n][2 * h + e], back[n][e], -ref[n][e]));
                    }
                if (__any_sync(0xffffffffu, over > room || step > top_step)) {
                    float shift = 0.f;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) step = fmaxf(step, __shfl_xor_sync(0xffffffffu, step, d));
                    if (step > top_step) {  // a power of two, so that the accumulators change by one too
                        const float now = __uint_as_float((__float_as_uint(step) & 0x7f800000u) + (5u << 23));
                        shift = (float)((int)(__float_as_uint(now) >> 23) - (int)(__float_as_uint(top_step) >> 23));
                        top_step = now, room -= shift;
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = -INFINITY;
#pragma unroll
                            for (int j = 0; j < kStepTiles; ++j) top = fmaxf(top, fmaxf(s[j][n][e], s[j][n][e + 2]) * back[n][e]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            float now = ref[n][e] + shift;
                            if (top - now > room) now = top + kSlack - room;
                            const float fall = exp2f(ref[n][e] - now);
                            ref[n][e] = now, sum[n][e] *= fall;
#pragma unroll
                            for (int i = 0; i < G; ++i) low[n][i][e] *= fall;
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) o[n][i][e] *= fall, o[n][i][e + 2] *= fall;
                        }
                }
#pragma unroll
                for (int j = 0; j < kStepTiles; ++j) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[j][n][e] = exp2_approx(fmaf(s[j][n][e], back[n][e & 1], -ref[n][e & 1]));
                            sum[n][e & 1] += s[j][n][e];
                        }
                    kvq_values<D, NT>(buf + j * Z::kStage + Z::kTileBytes, g, t, s[j], par[j], o, low);
                }
            }

            // ---- the unit is done, or this warp's share of it ----
            const bool begun = unit0 >= w0, ended = unit1 <= w1;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], d);
#pragma unroll
                    for (int i = 0; i < G; ++i)
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) low[n][i][e] += __shfl_xor_sync(0xffffffffu, low[n][i][e], d);
                }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][i][e] = fmaf(o[n][i][e], e < 2 ? 1.f : 0.0625f, low[n][i / 4][e & 1]);
            Part p{unit0, unit1, w.q.q0, row0, rows, head, 1};
            if (begun && ended) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float inv[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        inv[e] = sum[n][e] == 0.f ? 0.f : 1.f / sum[n][e];
                        if (a.lse && g == 0 && 8 * n + 2 * t + e < rows) store_lse(a, p, 8 * n + 2 * t + e, ref[n][e], sum[n][e]);
                    }
                    const int r = row0 + 8 * n + g;
                    uint16_t* dst = a.out.data + (int64_t)(w.q.q0 + r / a.group) * a.out.s_token +
                                    (int64_t)(head * a.group + r % a.group) * a.out.s_head + 2 * t;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {  // dims 16i + 8h + 2t, +1 of row g
                            const uint32_t y = transpose8(pack2(o[n][i][2 * h] * inv[0], o[n][i][2 * h + 1] * inv[1], a.bf != 0));
                            if (8 * n + g < rows) *reinterpret_cast<uint32_t*>(dst + 16 * i + 8 * h) = y;
                        }
                }
            } else {
                // a head part has a place of its own; a tail part ends the warp's share, so the ring is free
                float* at = begun ? reinterpret_cast<float*>(ring) : head_part;
                if (begun) {
                    cp_async_wait<0>();
                    __syncwarp();
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = 8 * n + 2 * t + e;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            at[r * Z::kPitch + 16 * i + g] = o[n][i][e];
                            at[r * Z::kPitch + 16 * i + 8 + g] = o[n][i][e + 2];
                        }
                        if (g == 0) at[RB * Z::kPitch + r] = ref[n][e], at[RB * Z::kPitch + RB + r] = sum[n][e];
                    }
                if (lane == 0) parts[wid][begun] = p;
            }
            unit0 = unit1;
            if (x < w1) next_unit<RB>(a, w);
        }
        cp_async_wait<0>();
    }
    __syncthreads();

    // ---- parts of one unit in this block ----
    uint32_t* counters = reinterpret_cast<uint32_t*>(a.workspace);
    float* slots = reinterpret_cast<float*>(a.workspace + kAttendCounterBytes);
    auto slot_of = [&](long long cta, int tail) { return slots + (2 * cta + tail) * Z::kSlotFloats; };
    if (tid < 2) last_of[tid] = 0;
    for (int w = -1; w < kWarps; ++w) {  // chains begin with the part that an earlier block began, or with a warp's tail
        if (w < 0 ? !parts[0][0].live : !parts[w][1].live) continue;
        const Part p = w < 0 ? parts[0][0] : parts[w][1];
        const int w_first = max(w, 0);
        int n = 1;
        while (w_first + n < kWarps && parts[w_first + n][0].live && parts[w_first + n][0].from == p.from) ++n;
        const bool alone = p.from >= cta0 && p.to <= cta1;
        const auto part = [&](int i) {
            return reinterpret_cast<const float*>(smem + (w_first + i) * Z::kWarpBytes + (w >= 0 && i == 0 ? 0 : Z::kRing));
        };
        if (alone) {
            merge<D, NT>(a, p, n, Z::kPitch, part, static_cast<float*>(nullptr));
        } else {
            const int tail = p.from >= cta0;
            merge<D, NT>(a, p, n, Z::kPitch, part, slot_of(blockIdx.x, tail));
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const long long first = p.from / per, last = (p.to - 1) / per;
                const bool all = atomicAdd(&counters[first], 1u) == (uint32_t)(last - first);
                if (all) counters[first] = 0;  // ready for the next call
                __threadfence();
                last_of[tail] = all;
            }
            __syncthreads();
            if (last_of[tail]) {
                const long long first = p.from / per;
                const auto slot = [&](int i) { return static_cast<const float*>(slot_of(first + i, i == 0)); };
                merge<D, NT>(a, p, (int)((p.to - 1) / per - first) + 1, D, slot, static_cast<float*>(nullptr));
            }
        }
    }
}

template <int D, int NT>
cudaError_t launch(AttendArgs& a, int sms, cudaStream_t stream) {
    using Z = Sizes<D, NT>;
    static_assert(Z::kBytes <= 227 * 1024, "shared memory");
    static_assert((size_t)2 * kAttendMaxCtas * Z::kSlotFloats * 4 + kAttendCounterBytes <= kAttendWorkspace, "workspace");
    const int per_sm = (D == 256 || NT == 2) ? 1 : 2;
    const int grid = std::min(sms * per_sm, kAttendMaxCtas);
    if (cudaError_t e = cudaFuncSetAttribute(kvq_attend_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Z::kBytes)) return e;
    kvq_attend_kernel<D, NT><<<grid, kThreads, Z::kBytes, stream>>>(a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

}  // namespace remp

using namespace remp;

extern "C" int64_t remp_kvq_workspace_bytes(void) { return (int64_t)kAttendWorkspace; }

extern "C" remp_status remp_kvq_attend(const remp_kvq_pool* pool, const remp_kvq_batch* batch, const remp_kvq_rows* q,
                                       const remp_kvq_rows* out, int32_t q_heads, int32_t dtype, float scale,
                                       int32_t window, float* lse, void* workspace, void* stream_) {
    AttendArgs a{};
    if (remp_status st = kvq_view(pool, batch, &a.v)) return st;
    if (dtype != REMP_DTYPE_BFLOAT && dtype != REMP_DTYPE_HALF) return fail(REMP_ERR_INVALID_ARG, "unknown dtype");
    if (q_heads < 1 || q_heads % pool->kv_heads) return fail(REMP_ERR_SHAPE, "q_heads must be a multiple of kv_heads");
    if (window < 0) return fail(REMP_ERR_INVALID_ARG, "negative window");
    if (!(scale > 0.f && scale <= 3.402823466e38f)) return fail(REMP_ERR_INVALID_ARG, "scale must be positive and finite");
    if (!workspace || (reinterpret_cast<uint64_t>(workspace) & 255))
        return fail(REMP_ERR_INVALID_ARG, "the workspace must be 256-byte aligned device memory");
    if (a.v.num_tokens == 0) return REMP_OK;
    if (batch->max_queries < 1) return fail(REMP_ERR_INVALID_ARG, "max_queries must be positive");
    if (remp_status st = kvq_rows(q, q_heads, pool->head_dim, "q", &a.q)) return st;
    if (remp_status st = kvq_rows(out, q_heads, pool->head_dim, "out", &a.out)) return st;
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    a.lse = lse, a.workspace = static_cast<uint8_t*>(workspace);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.group = q_heads / pool->kv_heads, a.q_heads = q_heads, a.window = window, a.bf = dtype == REMP_DTYPE_BFLOAT;
    a.spt = (a.v.num_seqs + kThreads - 1) / kThreads;
    if ((int64_t)batch->num_tokens * a.group > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "too many query rows");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool wide = (int64_t)batch->max_queries * a.group > 8;
    cudaError_t e;
    if (pool->head_dim == 64) e = wide ? launch<64, 2>(a, sms, stream) : launch<64, 1>(a, sms, stream);
    else if (pool->head_dim == 128) e = wide ? launch<128, 2>(a, sms, stream) : launch<128, 1>(a, sms, stream);
    else e = launch<256, 1>(a, sms, stream);
    if (e != cudaSuccess) return cuda_fail(e, "attention");
    return REMP_OK;
}
