// Attention over the 4-bit cache for few queries per sequence (decode, drafts, short continuations).
//
// Mathematics. With a key's codes c, step s and minimum m for each group of 64 dims, q.k = sum over groups of
// s*(q.c) + m*sum(q); with a value's, sum p*v = sum (p*s)*c + sum p*m. So the matrix instructions work on bare codes: a
// code in the low bits of a half is the subnormal c*2^-24, exact, and taking codes out of a word is an AND (and a shift for
// half of them); codes left at bits 4..7 count 16-fold, which the query's other half of the dims (K) or the output
// row (V) undoes. The factor 2^-24 leaves with the scale. Softmax with a running reference: the sums are kept
// relative to a reference that is raised by kSlack beyond a new maximum only when some score passes it (one vote per
// tile), so p <= 1 always and accumulators are seldom rescaled.
// Rounding: q is exact in half after a power of two per row; p*s is rounded to half (2^-11, before a sum of many); scores,
// references, sums of p, sums of p*m and outputs are in 32 bits.
//
// Roles: a tile is 16 tokens of one head. S^T[16 tokens][8 rows] = K.Q^T and O^T[D][8 rows] += V^T.P^T, so the eight query
// heads of a KV head fill the 8 columns of m16n8k16; P^T goes from accumulator to operand layout with one
// matrix transpose for each 8 tokens. NT = 2 takes 16 rows and is used when 8 do not hold a sequence's rows.
//
// Bound: HBM. Work is the list of all (sequence, row block, KV head, tile), cut evenly over the thread blocks and within
// one evenly over its warps, so ragged batches and single long sequences fill the GPU alike. A warp streams its
// tiles through a ring of kStages in shared memory with 16-byte asynchronous copies and needs no block-wide
// barrier until its share is done. Parts of a sequence are merged in the block, and across blocks by the block that
// arrives last (a counter; nobody waits), always in the order of the list: the result does not depend on timing.

#include "remp_kvq_device.h"

namespace remp {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr float kNoRef = -1e30f;  // reference of a row that has seen nothing; finite, so that -inf - kNoRef is -inf
constexpr float kSlack = 4.f;     // log2: a new reference is 16 times the maximum

struct AttendArgs {
    KvqView v;
    KvqRows q, out;
    float* lse;
    uint8_t* workspace;
    float scale_log2;  // softmax scale * log2(e)
    int32_t group, q_heads, window, bf;
    int32_t spt;       // sequences of one thread of the block-wide scan
    int32_t min_tiles; // tiles that a thread block takes at least
};

struct Seq {  // one sequence's share of the list
    int len, q0, rows;      // cached tokens, first row of the batch, query rows (queries * group)
    int tile0, tiles;       // tiles that its rows see; at least one, so that rows which see nothing are written too
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
    r.tiles = max(1, (r.len + kKvqTile - 1) / kKvqTile - r.tile0);
    return r;
}

template <int RB>
__device__ __forceinline__ long long tiles_of(const AttendArgs& a, int s) {
    const Seq q = seq_of<RB>(a, s);
    return (long long)q.blocks * a.v.kv_heads * q.tiles;
}

struct Cursor {  // a place in the list
    Seq q;
    int s, unit, tile;  // sequence, (KV head, row block) in it, tile in that
};

template <int RB>
__device__ __forceinline__ void next_unit(const AttendArgs& a, Cursor& c) {
    c.tile = 0;
    if (++c.unit < c.q.blocks * a.v.kv_heads) return;
    c.unit = 0;
    do {
        if (++c.s >= a.v.num_seqs) return;
        c.q = seq_of<RB>(a, c.s);
    } while (c.q.rows == 0);
}

struct Part {  // what a warp leaves of a unit that it did not see whole
    long long from, to;  // the unit's tiles in the list
    int q0, row0, rows, head;
    int live;
};

template <int D, int NT>
struct Sizes {
    static constexpr int kRows = 8 * NT;
    static constexpr int kTileBytes = kKvqTile * kvq_token_bytes(D);
    static constexpr int kStage = 2 * kTileBytes;
    static constexpr int kPitch = D + 4;                             // floats of a part's row: spreads the banks
    static constexpr int kPart = kRows * (kPitch + 2) * 4;           // rows, references, sums
    static constexpr int kStages = D == 256 ? 3 : 4;
    static constexpr int kRing = kStages * kStage > kPart ? kStages * kStage : kPart;  // the tail part reuses the ring
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
    constexpr int RB = Z::kRows, G = D / kKvqGroup, kStages = Z::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long scan[kThreads + 1];
    __shared__ long long warp_sum[kWarps];
    __shared__ Part parts[kWarps][2];
    __shared__ int last_of[2];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const KvqView& v = a.v;

    // ---- the list: tiles before each thread's sequences ----
    {
        long long mine = 0;
        const int s0 = min(v.num_seqs, tid * a.spt), s1 = min(v.num_seqs, s0 + a.spt);
        for (int s = s0; s < s1; ++s) {
            mine += tiles_of<RB>(a, s);
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
    const long long per = max((long long)a.min_tiles, (total + gridDim.x - 1) / gridDim.x);
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
        long long unit0;  // list index of tile 0 of the unit at work
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
                const long long n = (long long)c.q.blocks * v.kv_heads * c.q.tiles;
                if (at + n > w0) break;
                at += n;
            }
            const long long in = w0 - at;
            c.unit = (int)(in / c.q.tiles), c.tile = (int)(in % c.q.tiles);
            unit0 = w0 - c.tile;
        }
        Cursor w = c;

        // ---- loads: a ring of tiles, ids of 32 blocks at a time in the lanes ----
        int ids = -1, ids_seq = -1, ids_first = 0;
        uint32_t absent = 0;  // stages whose tile is not there
        auto issue = [&](int stage) {
            const int tile = c.q.tile0 + c.tile;
            const int in_row = tile / v.block_tiles;
            bool there = tile * kKvqTile < c.q.len;
            if (there) {
                if (c.s != ids_seq || in_row < ids_first || in_row >= ids_first + 32) {
                    ids_seq = c.s, ids_first = in_row;
                    ids = in_row + lane < v.max_blocks ? v.tables[(int64_t)c.s * v.max_blocks + in_row + lane] : -1;
                }
                const int id = __shfl_sync(0xffffffffu, ids, in_row - ids_first);
                there = id >= 0 && id < v.nb;
                if (there) {
                    const int head = c.unit / c.q.blocks;
                    const uint8_t* src = v.base + (int64_t)id * v.s_block + (int64_t)head * v.s_head +
                                         (tile - in_row * v.block_tiles) * Z::kTileBytes;
                    kvq_fetch_tile<D>(src, v.s_kv, ring_at + stage * Z::kStage, lane);
                } else if (lane == 0) {
                    kvq_error(v, kErrBadBlock);
                }
            }
            absent = there ? absent & ~(1u << stage) : absent | (1u << stage);
            if (++c.tile == c.q.tiles) next_unit<RB>(a, c);
        };
        long long ahead = w0;
        int load_stage = 0;
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) {
            if (ahead < w1) issue(load_stage), ++ahead;
            load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
            cp_async_commit();
        }

        // ---- work ----
        int stage = 0;
        for (long long x = w0; x < w1;) {
            const int head = w.unit / w.q.blocks, row0 = (w.unit - head * w.q.blocks) * RB;
            const int rows = min(RB, w.q.rows - row0);
            const long long unit1 = unit0 + w.q.tiles, stop = min(unit1, w1);

            // queries of this lane's column g (+8): halves of the operand, their sums, and the exponent that was taken out
            uint32_t qf[NT][D / 16][2];
            float qsum[NT][G][2], back[NT][2];
            int limit[NT][2];
            int low_limit = 0x7fffffff, high_limit = -1;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = row0 + min(8 * n + g, rows - 1);
                const bool real = 8 * n + g < rows;
                const uint16_t* src = a.q.data + (int64_t)(w.q.q0 + r / a.group) * a.q.s_token +
                                      (int64_t)(head * a.group + r % a.group) * a.q.s_head + 2 * t;
                kvq_load_queries<D>(src, a.bf != 0, real, t, qf[n], qsum[n], back[n], a.scale_log2);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = 8 * n + 2 * t + e;
                    limit[n][e] = col < rows ? w.q.first_pos + (row0 + col) / a.group : -1;
                }
                if (8 * n < rows) {
                    low_limit = min(low_limit, w.q.first_pos + (row0 + 8 * n) / a.group);
                    high_limit = max(high_limit, w.q.first_pos + (row0 + min(8 * n + 7, rows - 1)) / a.group);
                }
            }
            float o[NT][D / 16][4], ref[NT][2], sum[NT][2], low[NT][G][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
                ref[n][0] = ref[n][1] = kNoRef, sum[n][0] = sum[n][1] = 0.f;
#pragma unroll
                for (int i = 0; i < G; ++i) low[n][i][0] = low[n][i][1] = 0.f;
            }

            for (; x < stop; ++x) {
                cp_async_wait<kStages - 2>();
                __syncwarp();
                const uint8_t* buf = ring + stage * Z::kStage;
                const bool here = !(absent >> stage & 1);
                if (ahead < w1) issue(load_stage), ++ahead;
                load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
                cp_async_commit();
                stage = stage + 1 == kStages ? 0 : stage + 1;
                const int key0 = (w.q.tile0 + w.tile) * kKvqTile;
                ++w.tile;
                if (!here) continue;

                float s[NT][4];
                kvq_scores<D, NT>(buf, g, t, qf, qsum, s);
                const bool whole = key0 + kKvqTile - 1 <= low_limit && (a.window <= 0 || key0 > high_limit - a.window);
                if (!whole || key0 + kKvqTile > w.q.len) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + g + (e >> 1) * 8, lim = limit[n][e & 1];
                            if (key > lim || key >= w.q.len || (a.window > 0 && key <= lim - a.window)) s[n][e] = -INFINITY;
                        }
                }
                bool raise = false;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) raise |= s[n][e] * back[n][e & 1] > ref[n][e & 1];
                if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = fmaxf(s[n][e], s[n][e + 2]) * back[n][e];
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            if (top > ref[n][e]) {
                                const float fall = exp2f(ref[n][e] - (top + kSlack));
                                ref[n][e] = top + kSlack, sum[n][e] *= fall;
#pragma unroll
                                for (int i = 0; i < G; ++i) low[n][i][e] *= fall;
#pragma unroll
                                for (int i = 0; i < D / 16; ++i) o[n][i][e] *= fall, o[n][i][e + 2] *= fall;
                            }
                        }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[n][e] = exp2_approx(fmaf(s[n][e], back[n][e & 1], -ref[n][e & 1]));
                        sum[n][e & 1] += s[n][e];
                    }
                kvq_values<D, NT>(buf + Z::kTileBytes, g, t, s, key0 + kKvqTile > w.q.len, w.q.len - key0, o, low);
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
            // codes counted 2^-24 (2^-20 in the rows of the upper nibbles); add what the minima give
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[n][i][e] = fmaf(o[n][i][e], e < 2 ? 16777216.f : 1048576.f, low[n][i / 4][e & 1]);
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
    a.min_tiles = kWarps;
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
