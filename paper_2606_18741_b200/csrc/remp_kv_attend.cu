// Attention over a cache of 16-bit values for few queries per sequence (decode, drafts, short continuations).
//
// Mathematics: softmax with a running reference, p = 2^(x - ref). A reference moves only when a lane's sum of probabilities passes
// 2^room, by `slack` further than needed, which one vote for each tile finds out; accumulators are seldom rescaled. Sums of all
// lanes, warps and thread blocks stay below 1 in bfloat16, so that sums of p V stay below V's largest number, whatever that is.
// Rounding: a probability goes to the matrix instructions as two numbers of the cache's type, its first bits and what is left, so it
// keeps 16 bits and more (bfloat16 alone would give every probability an error of 2^-9); scores, references, sums and outputs are in
// 32 bits. The first is rounded towards 0 and the second is never 0, so that an infinity in V meets two numbers above 0
// and stays one.
//
// Roles: a tile is 16 tokens of one head. S^T[16 tokens][8 rows] = K.Q^T and O^T[D][8 rows] += V^T.P^T, so the eight query
// heads of a KV head fill the 8 columns of m16n8k16; P^T goes from accumulator to operand layout with one matrix transpose
// for each 8 tokens. NT = 2 takes 16 rows and is used when 8 do not hold a sequence's rows; 64 dims leave registers for 24 and 32.
//
// Bound: HBM. Work is the list of all (sequence, row block, KV head, tile), cut evenly over the thread blocks and within one evenly
// over its warps, so ragged batches and single long sequences fill the GPU alike. A warp streams its tiles through a ring in
// shared memory with 16-byte asynchronous copies, several tiles ahead, and needs no block-wide barrier until its share is
// done. The ring's 16-byte pieces change places within 8 rows (piece ^ (row & 7)), so matrix loads meet different banks. Rows
// that no query sees are not fetched but zeroed, so what their slots hold is never used. Parts of a sequence are merged in
// the block, and across blocks by the block that arrives last (a counter; nobody waits), in the order of the list.

#include "remp_attend_parts.h"
#include "remp_kv.h"
#include "remp_kv_attend.h"
#include "remp_kv_boxes.h"

namespace remp {

namespace {

// References. bfloat16: a lane's sum of all its probabilities stays at 2^-17; eight lanes, twelve warps and 512 thread blocks have at
// most 2^-1.4 of a row. A new reference puts the largest probability 14 powers of two below, far enough for most sequences
// (131072 tokens that weigh the same move it twice), and as p and V have the same exponents, nothing is lost on the way for V of
// 2^-70 and more. Half: its 2^-14 to 2^16 have to hold probabilities, and its largest V times 2^31 of them fits 32 bits, so only
// the sum of a tile is held below 2^14.
template <bool BF>
struct Refs {
    static constexpr float room = BF ? -17.f : 14.f, slack = BF ? 14.f : 4.f, bound = BF ? 0x1p-17f : 0x1p14f;
};

// Which kernel: this one takes up to 16 rows of a sequence (32 with 64 dims), and more where sequences and KV heads fill the GPU but are so
// short that a thread block for each costs more than it saves: this one takes a time for each tile and set of its rows, 1.4 ns for
// the whole GPU with 128 dims, 1.2 with 64, 4.1 with 256; the prompt kernel one for each tile, whatever the rows up to 256 (1.6, 1.6,
// 2.5), and for each sequence and KV head about 57, 42 and 46 more. Here and there, us in a graph, 8 KV heads: 128 dims, 20 rows, 1000
// sequences of 50 tokens 135 and 535, 300 of 500 242 and 266, 64 of 500 70 and 72, 24 of 3000 113 and 86, 2 of 16000 61 and 47; 64
// rows 254 and 553, 438 and 281, 119 and 78, 207 and 94, 98 and 51. 64 dims, 64 rows: 154 and 490, 213 and 258, 68 and 68, 109 and 84, 59
// and 43; 256 dims, 20 rows: 399 and 586, 674 and 342, 182 and 94, 322 and 131, 164 and 74. Where the GPU is not filled: 128 dims, 8
// of 400, 20 rows 25 and 18.
bool prompt_takes(int head_dim, int64_t rows, int64_t units, int sms, int64_t tokens) {
    const int set = head_dim == 64 ? 32 : 16;
    if (rows <= set) return false;
    if (units <= sms) return true;
    const int64_t sets = (rows + set - 1) / set, tiles = (tokens + kKvqTile - 1) / kKvqTile;
    return head_dim == 64 ? tiles * (5 * sets - 7) > 180 : head_dim == 128 ? tiles * (7 * sets - 8) > 290 : tiles * (5 * sets - 3) > 55;
}

struct Seq {  // one sequence's share of the list
    KvqSpan x;
    KvTiles tiles;
    int rows, blocks;  // query rows (queries * group), row blocks
    int steps;         // tiles; at least one, so that rows which see nothing are written too
};

template <int RB>
__device__ __forceinline__ Seq seq_of(const KvAttendArgs& a, int s) {
    Seq r;
    r.x = kvq_span(a.v.query_start[s], a.v.query_start[s + 1], a.v.seq_lens[s], a.v.num_tokens, a.room);
    r.rows = r.x.queries * a.group, r.blocks = (r.rows + RB - 1) / RB;
    r.tiles = kv_tiles(r.x, r.x.first_pos, a.window, a.first);
    r.steps = max(1, r.tiles.sinks + r.tiles.rest);
    return r;
}

struct Note {  // what the work on a step has to know; written by the loads
    int from, step, steps;         // the unit's first place in the list, the step of it, its steps
    int q0, row0, rows, head;      // rows [row0, row0 + rows) of the sequence whose first row is q0
    int first_pos, key0;
    uint32_t there;                // rows of the tile that some query sees
    int masked;                    // not every row sees every key
};

template <int D, int NT>
struct Sizes {
    static constexpr int kDim = D, kRows = 8 * NT, kQuads = NT * D / 16;
    static constexpr int kTile = kKvqTile * D * 2, kBuffer = 2 * kTile;  // K and V of a tile
    static constexpr int kStages = D == 64 ? (NT == 1 ? 4 : 3) : NT == 1 ? 3 : 2;
    // a part: accumulators as the lanes hold them (quad by quad), then references and sums of the rows
    static constexpr int kPartFloats = kQuads * 128 + 2 * kRows, kPart = kPartFloats * 4;
    static constexpr int kRing = kStages * kBuffer > kPart ? kStages * kBuffer : kPart;  // a tail part reuses the buffers
    static constexpr int kWarpBytes = (kRing + kPart + 63) / 64 * 64;
    // as many warps as there is room for, up to what their registers allow
    static constexpr int kMost = D == 64 ? (NT == 4 ? 8 : 12) : D == 128 ? 8 : 4, kFit = (227 * 1024 - 2304) / kWarpBytes;
    static constexpr int kWarps = kFit < kMost ? kFit : kMost, kThreads = kWarps * 32;
    static constexpr int kBytes = kWarps * kWarpBytes;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {  // not real: 16 bytes of zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
// Two probabilities' first bits, and what is left of them.
template <bool BF>
__device__ __forceinline__ uint32_t first2(float x, float y) {
    if (BF) return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
    uint32_t r;
    asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}
template <bool BF>
__device__ __forceinline__ uint32_t left2(float x, float y, uint32_t first) {
    if (BF) return pack2(fmaf(x, kAndMore, -bf_low(first)), fmaf(y, kAndMore, -bf_high(first)), true);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&first));
    return pack2(fmaxf(x - f.x, fminf(x, kLeastHalf)), fmaxf(y - f.y, fminf(y, kLeastHalf)), false);
}
__device__ __forceinline__ void load_matrices(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_transposed(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

template <int D, int NT, bool BF>
__global__ void __launch_bounds__(Sizes<D, NT>::kThreads, 1) kv_attend_kernel(const __grid_constant__ KvAttendArgs a) {
    using Z = Sizes<D, NT>;
    constexpr int RB = Z::kRows, kWarps = Z::kWarps, kThreads = Z::kThreads, kStages = Z::kStages, kPieces = D / 8;
    using Ref = Refs<BF>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long warp_sum[kWarps];
    __shared__ int first_at[kWarps], first_seq[kWarps];  // where a warp's share begins: sequences from here, at this place in the list
    __shared__ Unit parts[kWarps][2];  // of each warp: the unit that it found begun, the unit that it leaves unfinished
    __shared__ Chain chains[kWarps + 1];
    __shared__ int num_chains;
    __shared__ Note notes[kWarps][kStages];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const KvView& v = a.v;
    const int spt = (v.num_seqs + kThreads - 1) / kThreads;  // sequences of one thread in the scan
    grid_begin();

    // ---- the list: steps before each thread's sequences, and where this block's warps begin ----
    const int s0 = min(v.num_seqs, tid * spt), s1 = min(v.num_seqs, s0 + spt);
    long long mine = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const Seq q = seq_of<RB>(a, s);
        mine += (long long)q.blocks * v.kv_heads * q.steps;
        if (blockIdx.x == 0 && kvq_span_bad(q.x, v.seq_lens[s])) kvq_error(v, kErrBadLength);
    }
    long long before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += up;
    }
    if (lane == 31) warp_sum[wid] = before;
    if (tid < kWarps * 2) parts[tid >> 1][tid & 1].live = 0;
    __syncthreads();
    before -= mine;
    long long total_ = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const long long x = warp_sum[w];
        if (w < wid) before += x;
        total_ += x;
    }
    if (total_ > 0x40000000) {  // 2^30 tiles: more than 4 TB of cache
        if (blockIdx.x == 0 && tid == 0) kvq_error(v, kErrOverflow);
        return;
    }
    const int total = (int)total_, per = max(kWarps, (int)((uint32_t)(total + gridDim.x - 1) / gridDim.x));
    const int cta0 = min((long long)blockIdx.x * per, 0x7fffffffLL), cta1 = min(total, cta0 + per);
    if (cta0 >= total) return;
    const int wper = (cta1 - cta0 + kWarps - 1) / kWarps;
    if (mine > 0 && before < cta1 && before + mine > cta0) {
        // this thread's sequences hold the places [before, before + mine): the warps that begin there
        const int from = max(0, ((int)before - cta0 + wper - 1) / wper), to = (int)before + (int)mine - cta0;
#pragma unroll 1
        for (int w = from; w < kWarps && w * wper < to; ++w) first_seq[w] = s0, first_at[w] = (int)before;
    }
    __syncthreads();
    const int w0 = min(cta1, cta0 + wid * wper), todo = min(cta1, w0 + wper) - w0;

    uint8_t* const ring = smem + wid * Z::kWarpBytes;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);

    if (todo > 0) {
        // the loads' place in the list, kStages - 1 steps ahead of the work: sequence, KV head, row block, step of it
        Seq q{};
        int seq = first_seq[wid], seq_at = first_at[wid], head = 0, block = 0, step_at = 0;
        int ids = -1, in_ids = 32;      // ids of 32 blocks of the row of the table, one to a lane; the next tile's place among them
        int in_block = 0;               // its place in its block
        const uint8_t* heads = v.base;  // the KV head's rows of block 0
        const int32_t* row = nullptr;   // the rest of the row of the table
        int row_left = 0, low = 0, high = 0;  // positions of the unit's first and last row
        uint32_t qf[NT][D / 16][2];
        int limit[NT][2];               // positions of columns 2t, 2t + 1
        float o[NT][D / 16][4], ref[NT][2], sum[NT][2];
        bool fresh = true;              // the next step is the first of its unit here

#pragma unroll 1
        for (int i = 0; i < todo + kStages - 1; ++i) {
            if (i < todo) {
                // ---- loads of step i, into the buffer that the step kStages before it has left ----
                bool enter = i == 0;
                if (i > 0 && ++step_at == q.steps) {
                    step_at = 0, enter = true;
                    if (++block == q.blocks) block = 0, ++head;
                    if (head == v.kv_heads) head = 0, ++seq;
                }
                if (enter) {
                    if (i == 0 || (step_at | block | head) == 0) {
                        // the next sequence with rows; at first, the one that holds place w0
#pragma unroll 1
                        for (;; ++seq) {
                            q = seq_of<RB>(a, seq);
                            const int n = q.blocks * v.kv_heads * q.steps;
                            if (i == 0 ? seq_at + n > w0 : n > 0) break;
                            seq_at += n;
                        }
                    }
                    if (i == 0) {
                        const uint32_t in = w0 - seq_at, unit = in / (uint32_t)q.steps;
                        step_at = (int)(in - unit * q.steps), head = (int)(unit / (uint32_t)q.blocks), block = (int)unit - head * q.blocks;
                    }
                    heads = v.base + (int64_t)head * v.s_head;
                    // the unit's queries are wanted soon
                    const int r0 = block * RB, r = r0 + min(lane % RB, q.rows - r0 - 1), token = token_of(a, r);
                    const uint16_t* query = a.q.data + (int64_t)(q.x.q0 + token) * a.q.s_token + (int64_t)(head * a.group + r - token * a.group) * a.q.s_head;
                    for (int x = lane / RB * 64; lane < 32 / RB * RB && x < D; x += 32 / RB * 64) asm volatile("prefetch.global.L1 [%0];" ::"l"(query + x));
                    low = q.x.first_pos + token_of(a, r0), high = q.x.first_pos + token_of(a, min(r0 + RB, q.rows) - 1);
                }
                const int tile = step_at < q.tiles.sinks ? step_at : q.tiles.tile0 + step_at - q.tiles.sinks, key0 = tile * kKvqTile;
                if (enter || step_at == q.tiles.sinks) {  // another place in the row of the table
                    const int in_row = tile / v.block_tiles;
                    in_block = tile - in_row * v.block_tiles, in_ids = 32;
                    row = v.tables + (int64_t)seq * v.max_blocks + in_row, row_left = v.max_blocks - in_row;
                }
                uint32_t there = 0;
                int masked = 1;
                const uint8_t* src = heads;
                if (step_at < q.tiles.sinks + q.tiles.rest) {
                    if (in_ids == 32) {
                        ids = lane < row_left ? row[lane] : -1;
                        in_ids = 0, row += 32, row_left -= 32;
                    }
                    const int id = __shfl_sync(0xffffffffu, ids, in_ids);
                    if ((uint32_t)id < (uint32_t)v.nb) {
                        src = heads + (int64_t)id * v.s_block + (int64_t)in_block * kKvqTile * v.s_token;
                        masked = !(key0 + kKvqTile <= min(q.x.len, low + 1) && (key0 >= kvq_first_key(high, a.window) || key0 + kKvqTile <= a.first));
                        there = 0xffff;
                        if (masked) {
                            const int key = key0 + (lane & 15);
                            there = __ballot_sync(0xffffffffu, key < q.x.len && key <= high && (key >= kvq_first_key(low, a.window) || key < a.first)) & 0xffff;
                        }
                    } else if (lane == 0) {
                        kvq_error(v, kErrBadBlock);
                    }
                    if (++in_block == v.block_tiles) in_block = 0, ++in_ids;
                }
                const uint32_t dst = ring_at + i % kStages * Z::kBuffer;
#pragma unroll
                for (int x = 0; x < kKvqTile * kPieces / 32; ++x) {
                    const int r = lane / kPieces + x * (32 / kPieces), piece = lane % kPieces;
                    const bool real = there >> r & 1;
                    const uint8_t* from = real ? src + r * v.s_token + piece * 16 : v.base;
                    const uint32_t to = dst + r * (2 * D) + ((piece ^ (r & 7)) << 4);
                    copy16(to, from, real);
                    copy16(to + Z::kTile, real ? from + v.s_kv : from, real);
                }
                if (lane == 0)
                    notes[wid][i % kStages] = Note{w0 + i - step_at, step_at, q.steps, q.x.q0, block * RB, min(RB, q.rows - block * RB), head,
                                                   q.x.first_pos, key0, there, masked};
            }
            cp_async_commit();
            if (i < kStages - 1) continue;
            cp_async_wait<kStages - 1>();
            __syncwarp();

            // ---- work on step j ----
            const int j = i - (kStages - 1);
            const Note n = notes[wid][j % kStages];
            if (fresh) {  // the unit's queries: rows g (+8) are this lane's operand columns
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    const int r = n.row0 + min(8 * c + g, n.rows - 1), token = token_of(a, r);
                    kvq_load_queries<D>(a.q.data + (int64_t)(n.q0 + token) * a.q.s_token + (int64_t)(n.head * a.group + r - token * a.group) * a.q.s_head + 2 * t,
                                        8 * c + g < n.rows, qf[c]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        limit[c][e] = n.first_pos + token_of(a, n.row0 + min(8 * c + 2 * t + e, n.rows - 1));
                        ref[c][e] = kNoRef, sum[c][e] = 0.f;
                    }
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) o[c][k][0] = o[c][k][1] = o[c][k][2] = o[c][k][3] = 0.f;
                }
                fresh = false;
            }
            const uint32_t buf = ring_at + j % kStages * Z::kBuffer;
            float s[NT][4];
            {
                float even[NT][4], odd[NT][4];  // two chains
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) even[c][e] = odd[c][e] = 0.f;
                const uint32_t at = buf + (lane & 15) * (2 * D), swap = ((lane >> 4) ^ (lane & 7)) << 4;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    uint32_t x[4];
                    load_matrices(at + (swap ^ (k * 32)), x);
#pragma unroll
                    for (int c = 0; c < NT; ++c) mma_rows<BF>(k & 1 ? odd[c] : even[c], x, qf[c][k][0], qf[c][k][1]);
                }
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[c][e] = (even[c][e] + odd[c][e]) * a.scale_log2;
            }
            if (n.masked) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int key = n.key0 + g + 8 * h;
                    const bool there = n.there >> (g + 8 * h) & 1;
#pragma unroll
                    for (int c = 0; c < NT; ++c)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (!there || !kv_sees(limit[c][e], key, a.window, a.first)) s[c][2 * h + e] = -INFINITY;
                }
            }
            // probabilities against the references as they are, or against higher ones where their sums pass the room
            float p[NT][4], held[NT][2];  // held: the sums with this tile; half: of this tile
#pragma unroll 1
            for (int round = 0;; ++round) {
                float most = 0.f;
#pragma unroll
                for (int c = 0; c < NT; ++c) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[c][e] = exp2_approx(s[c][e] - ref[c][e & 1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) held[c][e] = p[c][e] + p[c][e + 2] + (BF ? sum[c][e] : 0.f);
                    most = max3(most, held[c][0], held[c][1]);
                }
                if (round || !__any_sync(0xffffffffu, most > Ref::bound)) break;
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(s[c][e], s[c][e + 2]), all = held[c][e];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1)
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d)), all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, d));
                        float now = ref[c][e];
                        if (all > Ref::bound) now = fmaxf(top + Ref::slack - Ref::room, BF ? now + Ref::slack : now);
                        const float fall = exp2_approx(ref[c][e] - now);
                        ref[c][e] = now, sum[c][e] *= fall;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) o[c][k][e] *= fall, o[c][k][e + 2] *= fall;
                    }
            }
            uint32_t high_p[NT][2], low_p[NT][2];
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                sum[c][0] = BF ? held[c][0] : sum[c][0] + held[c][0], sum[c][1] = BF ? held[c][1] : sum[c][1] + held[c][1];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t first = first2<BF>(p[c][2 * h], p[c][2 * h + 1]);
                    high_p[c][h] = transpose8(first), low_p[c][h] = transpose8(left2<BF>(p[c][2 * h], p[c][2 * h + 1], first));
                }
            }
            {
                const uint32_t at = buf + Z::kTile + ((lane & 7) + (lane >> 4) * 8) * (2 * D), swap = ((lane >> 3 & 1) ^ (lane & 7)) << 4;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    uint32_t x[4];
                    load_transposed(at + (swap ^ (k * 32)), x);
#pragma unroll
                    for (int c = 0; c < NT; ++c) mma_rows<BF>(o[c][k], x, high_p[c][0], high_p[c][1]), mma_rows<BF>(o[c][k], x, low_p[c][0], low_p[c][1]);
                }
            }
            __syncwarp();  // the buffer and the note are read

            const bool ended = n.step + 1 == n.steps;
            if (!ended && j + 1 < todo) continue;
            // ---- the unit is done, or this warp's share of it ----
            const bool begun = n.from >= w0;
            const Unit u{n.from, n.from + n.steps, n.q0, n.row0, n.rows, n.head, 1};
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) sum[c][e] += __shfl_xor_sync(0xffffffffu, sum[c][e], d);
            const auto quad = [&](int c, int k) { return make_float4(o[c][k][0], o[c][k][1], o[c][k][2], o[c][k][3]); };
            if (begun && ended) {
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    const float inv[2] = {sum[c][0] == 0.f ? 0.f : 1.f / sum[c][0], sum[c][1] == 0.f ? 0.f : 1.f / sum[c][1]};
                    if (a.lse && g == 0) put_lse(a, u, 8 * c + 2 * t, ref[c][0], sum[c][0]), put_lse(a, u, 8 * c + 2 * t + 1, ref[c][1], sum[c][1]);
                    uint16_t* dst = out_row(a, u, c, g, t);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) put_quad<BF>(quad(c, k), inv, dst + 16 * k, 8 * c + g < u.rows);
                }
            } else {
                // a head part has a place of its own; a tail part ends the warp's share, so the buffers are free
                float* at = reinterpret_cast<float*>(ring + (begun ? 0 : Z::kRing));
#pragma unroll
                for (int c = 0; c < NT; ++c) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) *reinterpret_cast<float4*>(at + (c * (D / 16) + k) * 128 + lane * 4) = quad(c, k);
                    if (g == 0) {
                        *reinterpret_cast<float2*>(at + Z::kQuads * 128 + 8 * c + 2 * t) = make_float2(ref[c][0], ref[c][1]);
                        *reinterpret_cast<float2*>(at + Z::kQuads * 128 + RB + 8 * c + 2 * t) = make_float2(sum[c][0], sum[c][1]);
                    }
                }
                if (lane == 0) parts[wid][begun] = u;
            }
            fresh = true;
        }
    }
    merge_parts<Z, BF>(a, smem, parts, chains, &num_chains, cta0, cta1, per);
}

template <int D, int NT>
cudaError_t launch(const KvAttendArgs& a, bool bf, int sms, cudaStream_t stream) {
    using Z = Sizes<D, NT>;
    static_assert(Z::kBytes + 2304 <= 227 * 1024, "shared memory");  // and what the kernel has beside it
    static_assert((size_t)2 * kAttendMaxCtas * Z::kPart + kAttendCounterBytes <= kAttendWorkspace, "workspace");
    const int grid = std::min(sms, kAttendMaxCtas);
    return launch_after(bf ? kv_attend_kernel<D, NT, true> : kv_attend_kernel<D, NT, false>, grid, Z::kThreads, Z::kBytes, stream, a);
}

// With room for the rows of the longest sequence of queries, up to NT times 8.
template <int D, int NT>
cudaError_t launch_rows(const KvAttendArgs& a, int64_t rows, bool bf, int sms, cudaStream_t stream) {
    if constexpr (NT > 1)
        if (rows <= 8 * (NT - 1)) return launch_rows<D, NT - 1>(a, rows, bf, sms, stream);
    return launch<D, NT>(a, bf, sms, stream);
}

}  // namespace

}  // namespace remp

using namespace remp;

extern "C" int64_t remp_kv_workspace_bytes(void) { return (int64_t)kAttendWorkspace; }

extern "C" remp_status remp_kv_attend(const remp_kv_pool* pool, const remp_kvq_batch* batch, const remp_kvq_rows* q,
                                      const remp_kvq_rows* out, int32_t q_heads, int32_t dtype, float scale, int32_t window,
                                      int32_t first, float* lse, void* workspace, void* stream_) {
    KvAttendArgs a{};
    if (remp_status st = kv_view(pool, batch, &a.v)) return st;
    if (remp_status st = kvq_dtype(dtype)) return st;
    if (remp_status st = kv_mask(scale, window, first)) return st;
    if (remp_status st = kv_group(q_heads, pool->kv_heads, batch->num_tokens, &a.group, &a.by_group)) return st;
    if (!workspace || (reinterpret_cast<uint64_t>(workspace) & 255))
        return fail(REMP_ERR_INVALID_ARG, "the workspace must be 256-byte aligned device memory");
    if (a.v.num_tokens == 0) return REMP_OK;
    if (batch->max_queries < 1) return fail(REMP_ERR_INVALID_ARG, "max_queries must be positive");
    if (remp_status st = kvq_rows(q, a.v.num_tokens, q_heads, pool->head_dim, false, "q", &a.q)) return st;
    if (remp_status st = kvq_rows(out, a.v.num_tokens, q_heads, pool->head_dim, true, "out", &a.out)) return st;
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    a.lse = lse, a.workspace = static_cast<uint8_t*>(workspace);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.q_heads = q_heads, a.window = window, a.first = window > 0 ? first : 0;
    a.room = (int32_t)std::min<int64_t>((int64_t)a.v.max_blocks * a.v.block_tiles * kKvqTile, kKvqMost);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int64_t max_rows = (int64_t)std::min(batch->max_queries, batch->num_tokens) * a.group;
    const bool bf = dtype == REMP_DTYPE_BFLOAT;
    cudaError_t e;
    // cached tokens that a sequence's rows see at most, as far as the host knows
    const int64_t seen = window > 0 ? std::min<int64_t>(a.room, (int64_t)window + a.first + batch->max_queries) : a.room;
    if (prompt_takes(pool->head_dim, max_rows, (int64_t)a.v.num_seqs * pool->kv_heads, sms, seen) && kv_boxes_take(a.v)) e = launch_kv_prompt(a, pool->head_dim, bf, sms, (int32_t)max_rows, stream);
    else if (pool->head_dim == 64) e = launch_rows<64, 4>(a, max_rows, bf, sms, stream);
    else if (pool->head_dim == 128) e = launch_rows<128, 2>(a, max_rows, bf, sms, stream);
    else e = launch_rows<256, 2>(a, max_rows, bf, sms, stream);
    if (e != cudaSuccess) return cuda_fail(e, "attention");
    return REMP_OK;
}
