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
// Measured: 64 query and 8 KV heads over about 100 thousand tokens of 29 sequences (114.5 MB) 44 us, 2.6 TB/s; 40 query
// heads over 131071 tokens (151 MB) 50 us, 3.0 TB/s; 2048 sequences of 1 to 63 tokens (71.6 MB) 41 us. Not bound by HBM:
// the long case, profiled just before its last step (57 us in the profile), took 404 instructions for a tile's K and V, with
// the integer pipe at 54 %, issue slots at 56 % and the tensor pipe at 18 %.

#include "remp_attend_parts.h"
#include "remp_kvq_device.h"

namespace remp {

namespace {

constexpr float kSlack = 4.f;     // log2: a new reference leaves room for scores up to 4 higher and steps up to 16 times larger
// Steps below this are not looked at: p stays at or below 2^45, so that p*m of groups without a step (m up to 2^60 and more) and
// their sums fit, and p*s of steps down to 2^-50 keeps its bits.
constexpr float kTopStep = 0x1p-30f, kTopBound = 0x1p45f;
// Rows up to which this kernel takes a sequence; above, the prompt kernel. Prompt / this one, us in a graph: rows x sequences x
// keys, 8 KV heads of 128 dims, 4 to 8 query heads for each: 24 x 16 x 2000 48.4 / 43.1, 20 x 64 x 500 69.8 / 51.3; 40 x 8 x
// 4000 51.4 / 55.4, 64 x 64 x 1000 108.7 / 129.3.
constexpr int kPromptRows = 32;
constexpr int kStepTiles = 2, kStepTokens = kStepTiles * kKvqTile;

struct AttendArgs {
    KvqView v;
    KvqRows q, out;
    float* lse;
    uint8_t* workspace;
    float scale_log2;  // softmax scale * log2(e)
    int32_t group, q_heads, window;
    uint32_t by_group; // row / group = high half of row * by_group (0: group is 1)
    int32_t room;      // tokens that a row of the table holds
};

struct Seq {  // one sequence's share of the list
    int len, q0, rows;      // cached tokens, first row of the batch, query rows (queries * group)
    int tile0, tiles;       // tiles that its rows see
    int steps;              // of kStepTiles; at least one, so that rows which see nothing are written too
    int first_pos;          // position of its first query
    int blocks;             // row blocks
    bool bad;               // the length was cut, or a row stands before position 0
};

template <int RB>
__device__ __forceinline__ Seq seq_of(const AttendArgs& a, int s) {
    Seq r;
    const int length = a.v.seq_lens[s];
    const KvqSpan x = kvq_span(a.v.query_start[s], a.v.query_start[s + 1], length, a.v.num_tokens, a.room);
    r.bad = kvq_span_bad(x, length);
    r.len = x.len, r.q0 = x.q0, r.first_pos = x.first_pos;
    r.rows = x.queries * a.group, r.blocks = (r.rows + RB - 1) / RB;
    r.tile0 = min(kvq_first_key(x.first_pos, a.window), x.len) / kKvqTile;
    r.tiles = (r.len + kKvqTile - 1) / kKvqTile - r.tile0;
    r.steps = max(1, (r.tiles + kStepTiles - 1) / kStepTiles);
    return r;
}

template <int D, int NT>
struct Sizes {
    // One block to an SM: twelve warps of 168 registers hold everything where eight rows of up to 128 dims are at work (70B decode
    // step 46 us, 131071 tokens 53 us; two blocks of eight warps, which spill: 52 and 65; three of four: 48 and 75), eight
    // of 255 elsewhere.
    static constexpr int kWarps = D == 256 || NT == 2 ? 8 : 12, kThreads = kWarps * 32;
    static constexpr int kDim = D, kRows = 8 * NT, kQuads = NT * D / 16;
    static constexpr int kTileBytes = kKvqTile * kvq_token_bytes(D);
    static constexpr int kBuffer = KvqStep<D>::kBytes;
    // a part: accumulators as the lanes hold them (quad by quad), then references and sums of the rows
    static constexpr int kPartFloats = kQuads * 128 + 2 * kRows, kPart = kPartFloats * 4;
    static constexpr int kRing = 2 * kBuffer > kPart ? 2 * kBuffer : kPart;  // a tail part reuses the buffers
    static constexpr int kWarpBytes = (kRing + kPart + 127) / 128 * 128;
    static constexpr int kBytes = kWarps * kWarpBytes;
};

template <int D, int NT, bool BF>
__global__ void __launch_bounds__(Sizes<D, NT>::kThreads, 1) kvq_attend_kernel(const __grid_constant__ AttendArgs a) {
    using Z = Sizes<D, NT>;
    using S = KvqStep<D>;
    constexpr int RB = Z::kRows, G = D / kKvqGroup, kWarps = Z::kWarps, kThreads = Z::kThreads;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long warp_sum[kWarps];
    __shared__ int first_at[kWarps], first_seq[kWarps];  // where a warp's share begins: sequences from here, at this place in the list
    __shared__ Unit parts[kWarps][2];  // of each warp: the unit that it found begun, the unit that it leaves unfinished
    __shared__ Chain chains[kWarps + 1];
    __shared__ int num_chains;

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const KvqView& v = a.v;
    const int spt = (v.num_seqs + kThreads - 1) / kThreads;  // sequences of one thread in the scan
    grid_begin();

    // ---- the list: steps before each thread's sequences, and where this block's warps begin ----
    const int s0 = min(v.num_seqs, tid * spt), s1 = min(v.num_seqs, s0 + spt);
    long long mine = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const Seq q = seq_of<RB>(a, s);
        mine += (long long)(q.blocks * v.kv_heads) * q.steps;
        if (blockIdx.x == 0 && q.bad) kvq_error(v, kErrBadLength);
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
    if (total_ > 0x40000000) {  // 2^30 steps: more than 4 TB of cache
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

    uint8_t* ring = smem + wid * Z::kWarpBytes;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);

    if (todo > 0) {
        // the loads' place in the list, one step ahead of the work: sequence, KV head, row block, step of it
        Seq q{};
        int seq = first_seq[wid], seq_at = first_at[wid], head = 0, block = 0, step_at = 0;
        int ids = -1, in_ids = 32;    // ids of 32 blocks of the row of the table, one to a lane; the next tile's place among them
        int in_block = 0;             // its place in its block
        const uint8_t* heads = v.base;  // the KV head's slice of block 0
        const int32_t* row = nullptr;   // the rest of the row of the table
        int row_left = 0;
        uint32_t absent = 0;                        // tiles of the step that are not there
        uint32_t qf[NT][D / 16][2];
        float qsum[NT][G][2], back[NT][2];
        int limit[NT][2];  // positions of columns 2t, 2t+1
        float o[NT][D / 16][4], ref[NT][2], sum[NT][2], low[NT][G][2];
        float top_step = kTopStep, bound = kTopBound;  // p * top_step <= 2^15: p <= bound
        uint32_t lift = 0;                       // columns whose scores take the 2^20 that `back` does not hold, bit 2n + e
        bool fresh = true;                       // the next step is the first of its unit here

#pragma unroll 1
        for (int i = 0; i <= todo; ++i) {
            cp_async_wait<0>();
            __syncwarp();
            // the step at work is the one that was asked for in the last round
            const uint32_t missing = absent;
            const Seq wq = q;
            const int w_head = head, w_block = block, w_step = step_at;
            if (i < todo) {
                // ---- loads of step i, into the buffer that the step before the last has left ----
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
                    const int tile = q.tile0 + step_at * kStepTiles, in_row = tile / v.block_tiles;
                    in_block = tile - in_row * v.block_tiles, in_ids = 32;
                    row = v.tables + (int64_t)seq * v.max_blocks + in_row, row_left = v.max_blocks - in_row;
                    heads = v.base + (int64_t)head * v.s_head;
                    // the unit's queries are wanted in the next round
                    const int r0 = block * RB, r = r0 + min(lane & (RB - 1), q.rows - r0 - 1), token = token_of(a, r);
                    const uint16_t* query = a.q.data + (int64_t)(q.q0 + token) * a.q.s_token + (int64_t)(head * a.group + r - token * a.group) * a.q.s_head;
                    for (int x = lane / RB * 64; x < D; x += 32 / RB * 64) asm volatile("prefetch.global.L1 [%0];" ::"l"(query + x));
                }
                const int left = q.tiles - step_at * kStepTiles;
                const auto tile_at = [&](const uint8_t*& src) {  // of the next tile; false: its block is not in the pool
                    if (in_ids == 32) {
                        ids = lane < row_left ? row[lane] : -1;
                        in_ids = 0, row += 32, row_left -= 32;
                    }
                    const int id = __shfl_sync(0xffffffffu, ids, in_ids);
                    src = heads + (int64_t)id * v.s_block + in_block * Z::kTileBytes;
                    if (++in_block == v.block_tiles) in_block = 0, ++in_ids;
                    const bool there = (uint32_t)id < (uint32_t)v.nb;
                    if (!there && lane == 0) kvq_error(v, kErrBadBlock);
                    return there;
                };
                const uint8_t *src0 = heads, *src1 = heads;
                const bool there0 = left > 0 && tile_at(src0), there1 = left > 1 && tile_at(src1);
                absent = (there0 ? 0u : 1u) | (there1 ? 0u : 2u);
                kvq_fetch_step<D>(src0, src1, there0, there1, v.s_kv, ring_at + (i & 1) * Z::kBuffer, lane);
            }
            cp_async_commit();
            if (i == 0) continue;

            // ---- work on step i - 1 ----
            if (fresh) {  // the unit's queries: rows g (+8) are this lane's operand columns
                const int row0 = w_block * RB, rows = wq.rows - row0;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int r = row0 + min(8 * n + g, rows - 1), token = token_of(a, r);
                    kvq_load_queries<D>(a.q.data + (int64_t)(wq.q0 + token) * a.q.s_token +
                                            (int64_t)(w_head * a.group + r - token * a.group) * a.q.s_head + 2 * t,
                                        8 * n + g < rows, qf[n]);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    kvq_make_queries<D>(BF, t, qf[n], qsum[n], back[n], a.scale_log2);
                    lift = n ? lift : 0;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (back[n][e] < 0.f) lift |= 1u << (2 * n + e), back[n][e] = -back[n][e];
                        limit[n][e] = wq.first_pos + token_of(a, row0 + min(8 * n + 2 * t + e, rows - 1));
                        ref[n][e] = kNoRef, sum[n][e] = 0.f;
#pragma unroll
                        for (int j = 0; j < G; ++j) low[n][j][e] = 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) o[n][j][0] = o[n][j][1] = o[n][j][2] = o[n][j][3] = 0.f;
                }
                top_step = kTopStep, bound = kTopBound, fresh = false;
            }
            const uint8_t* buf = ring + ((i - 1) & 1) * Z::kBuffer;
            const int key0 = (wq.tile0 + w_step * kStepTiles) * kKvqTile;
            float s[kStepTiles][NT][4];
            uint32_t par[kStepTiles][2][G];
#pragma unroll
            for (int j = 0; j < kStepTiles; ++j) {
                kvq_scores<D, NT>(buf + S::kK + j * S::kCodes, buf + S::kParK + j * S::kParams, g, t, qf, qsum, s[j]);
                kvq_params<D>(buf + S::kParV + j * S::kParams, g, par[j]);
            }
            if (__any_sync(0xffffffffu, lift != 0)) {
#pragma unroll
                for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (lift >> (2 * n + (e & 1)) & 1) s[j][n][e] *= 1048576.f;
            }
            if (missing || key0 + kStepTokens > wq.len || key0 + kStepTokens - 1 > wq.first_pos || a.window > 0) {
                // what a row does not see gets -infinity; the steps and minima of tokens that are not there, 0
#pragma unroll
                for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int key = key0 + j * kKvqTile + g + 8 * h;
                        const bool there = key < wq.len && !(missing >> j & 1);
#pragma unroll
                        for (int k = 0; k < G; ++k)
                            if (!there) par[j][h][k] = 0;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (!there || key > limit[n][e] || (a.window > 0 && limit[n][e] - key >= a.window))
                                    s[j][n][2 * h + e] = -INFINITY;
                    }
            }
            // probabilities against the references as they are; none above 2^room if their sums are not
            float p[kStepTiles][NT][4], tsum[NT][2], step = 0.f;
#pragma unroll
            for (int k = 0; k < G; ++k) {
                step = max3(step, bf_low(par[0][0][k]), bf_low(par[0][1][k]));
                step = max3(step, bf_low(par[1][0][k]), bf_low(par[1][1][k]));
            }
#pragma unroll 1
            for (int round = 0;; ++round) {
                float most = 0.f;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[j][n][e] = exp2_approx(fmaf(s[j][n][e], back[n][e & 1], -ref[n][e & 1]));
#pragma unroll
                    for (int e = 0; e < 2; ++e) tsum[n][e] = (p[0][n][e] + p[0][n][e + 2]) + (p[1][n][e] + p[1][n][e + 2]);
                    most = max3(most, tsum[n][0], tsum[n][1]);
                }
                if (round || !__any_sync(0xffffffffu, most > bound || step > top_step)) break;
                int shift = 0;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) step = fmaxf(step, __shfl_xor_sync(0xffffffffu, step, d));
                if (step > top_step) {  // a power of two, so that the accumulators change by one too
                    const float now = __uint_as_float((__float_as_uint(step) & 0x7f800000u) + (5u << 23));
                    shift = (int)(__float_as_uint(now) >> 23) - (int)(__float_as_uint(top_step) >> 23);
                    top_step = now, bound = __uint_as_float(__float_as_uint(bound) - ((uint32_t)shift << 23));
                }
                const float room = (float)((int)(__float_as_uint(bound) >> 23) - 127);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(fmaxf(s[0][n][e], s[0][n][e + 2]), fmaxf(s[1][n][e], s[1][n][e + 2])) * back[n][e];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        float now = ref[n][e] + (float)shift;
                        if (top - now > room - 2.f) now = top + kSlack - room;  // four of them may be this large
                        const float fall = exp2_approx(ref[n][e] - now);
                        ref[n][e] = now, sum[n][e] *= fall;
#pragma unroll
                        for (int k = 0; k < G; ++k) low[n][k][e] *= fall;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) o[n][k][e] *= fall, o[n][k][e + 2] *= fall;
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) sum[n][0] += tsum[n][0], sum[n][1] += tsum[n][1];
#pragma unroll
            for (int j = 0; j < kStepTiles; ++j) kvq_values<D, NT>(buf + S::kV + j * S::kCodes, g, t, p[j], par[j], o, low);

            const bool ended = w_step + 1 == wq.steps;
            if (!ended && i < todo) continue;
            // ---- the unit is done, or this warp's share of it ----
            const int unit0 = w0 + i - 1 - w_step;
            const bool begun = unit0 >= w0;
            const Unit u{unit0, unit0 + wq.steps, wq.q0, w_block * RB, min(RB, wq.rows - w_block * RB), w_head, 1};
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], d);
#pragma unroll
                    for (int k = 0; k < G; ++k)
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) low[n][k][e] += __shfl_xor_sync(0xffffffffu, low[n][k][e], d);
                }
            const auto quad = [&](int n, int k) {
                return make_float4(o[n][k][0] + low[n][k / 4][0], o[n][k][1] + low[n][k / 4][1],
                                   fmaf(o[n][k][2], 0.0625f, low[n][k / 4][0]), fmaf(o[n][k][3], 0.0625f, low[n][k / 4][1]));
            };
            if (begun && ended) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float inv[2] = {sum[n][0] == 0.f ? 0.f : 1.f / sum[n][0], sum[n][1] == 0.f ? 0.f : 1.f / sum[n][1]};
                    if (a.lse && g == 0) put_lse(a, u, 8 * n + 2 * t, ref[n][0], sum[n][0]), put_lse(a, u, 8 * n + 2 * t + 1, ref[n][1], sum[n][1]);
                    uint16_t* dst = out_row(a, u, n, g, t);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) put_quad<BF>(quad(n, k), inv, dst + 16 * k, 8 * n + g < u.rows);
                }
            } else {
                // a head part has a place of its own; a tail part ends the warp's share, so the buffers are free
                float* at = reinterpret_cast<float*>(ring + (begun ? 0 : Z::kRing));
                __syncwarp();
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) *reinterpret_cast<float4*>(at + (n * (D / 16) + k) * 128 + lane * 4) = quad(n, k);
                    if (g == 0) {
                        *reinterpret_cast<float2*>(at + Z::kQuads * 128 + 8 * n + 2 * t) = make_float2(ref[n][0], ref[n][1]);
                        *reinterpret_cast<float2*>(at + Z::kQuads * 128 + RB + 8 * n + 2 * t) = make_float2(sum[n][0], sum[n][1]);
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
cudaError_t launch(const AttendArgs& a, bool bf, int sms, cudaStream_t stream) {
    using Z = Sizes<D, NT>;
    static_assert(Z::kBytes <= 222 * 1024, "shared memory");
    static_assert((size_t)2 * kAttendMaxCtas * Z::kPart + kAttendCounterBytes <= kAttendWorkspace, "workspace");
    const int grid = std::min(sms, kAttendMaxCtas);
    return launch_after(bf ? kvq_attend_kernel<D, NT, true> : kvq_attend_kernel<D, NT, false>, grid, Z::kThreads, Z::kBytes, stream, a);
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
    if (remp_status st = kvq_rows(q, a.v.num_tokens, q_heads, pool->head_dim, false, "q", &a.q)) return st;
    if (remp_status st = kvq_rows(out, a.v.num_tokens, q_heads, pool->head_dim, true, "out", &a.out)) return st;
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    a.lse = lse, a.workspace = static_cast<uint8_t*>(workspace);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.group = q_heads / pool->kv_heads, a.q_heads = q_heads, a.window = window;
    a.room = (int32_t)std::min<int64_t>((int64_t)a.v.max_blocks * a.v.block_tiles * kKvqTile, kKvqMost);
    // rows are divided by the group with one multiplication: exact while row * group stays below 2^32
    if ((int64_t)batch->num_tokens * a.group * a.group > 0x7fffffffLL) return fail(REMP_ERR_SHAPE, "too many query rows");
    a.by_group = a.group == 1 ? 0 : (uint32_t)((0x100000000ULL + a.group - 1) / a.group);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int64_t max_rows = (int64_t)std::min(batch->max_queries, batch->num_tokens) * a.group;
    const bool bf = dtype == REMP_DTYPE_BFLOAT, wide = max_rows > 8;
    cudaError_t e;
    if (max_rows > kPromptRows)
        e = launch_prompt(a.v, a.q, a.out, lse, workspace, a.scale_log2, pool->head_dim, q_heads, a.group, a.by_group, window, a.room, bf, sms,
                          (int32_t)max_rows, stream);
    else if (pool->head_dim == 64) e = wide ? launch<64, 2>(a, bf, sms, stream) : launch<64, 1>(a, bf, sms, stream);
    else if (pool->head_dim == 128) e = wide ? launch<128, 2>(a, bf, sms, stream) : launch<128, 1>(a, bf, sms, stream);
    else e = launch<256, 1>(a, bf, sms, stream);
    if (e != cudaSuccess) return cuda_fail(e, "attention");
    return REMP_OK;
}
