// Attention over a cache of 16-bit values for many queries per sequence (prompts and their chunks, drafts of wide groups), on the tensor
// cores' own memory.
//
// Mathematics: softmax(scale * q.K^T + mask).V, one thread block for 256 rows (tokens x query heads of one KV head; two
// matrices of 128) and a range of the keys, block by block of kKeys keys: S = Q.K^T, P = 2^(S*scale - ref), O += P.V, with a
// running reference for each row that moves only when its probabilities outgrow a bound.
// Rounding: the matrix instructions take P in the cache's type only. Up to 64 rows (drafts, wide groups, single tokens beside a
// prompt) fill no more than half of a matrix: the other half takes the same rows, and where lane r has the first bits of a
// probability, lane 64 + r has what is left of it, so it keeps 16 bits and more at no cost in instructions; the two products are added
// at the end. More rows round it (bfloat16: by 2^-9 at most, an error of 0.0023 against 64 bits where 16 bits have 0.0017): a second
// product of every block with what makes its operand took 524 us in place of 424 in the case below. S, O, sums and references are in
// 32 bits.
//
// Bound: tensor cores (4*D flops for each row and key) and, as closely, the exponentials (one for each row and key; 16 a cycle of an
// SM). Eight warps compute P (a row to a thread), one thread issues the matrix instructions, which run for one matrix while P of the
// other is made, one warp brings K and V. Q and a ring of blocks of K and of V lie in shared memory in rows of 128 bytes, 16-byte
// pieces exchanged within 8 rows (piece ^ (row & 7)), as bulk tensor copies of a tile bring them: the keys of a block are rows
// of B along the dims for S and across them for O, so nothing is transposed. S and P share their columns of the tensor memory, O
// has its own; P goes to the matrix instructions in two parts, so that the products of three quarters of a block run while the last
// is made. With 256 dims O takes so much of it that one matrix of 128 rows and blocks of 64 keys are left.
//
// Measured, 2 x 2048 queries of 32 heads over 8191 tokens of 4 KV heads, 128 dims (us in a graph): 752 with 16-byte copies by three
// warps; 570 with boxes of 64 dims; 553 with one thread that waits and issues (a warp took 200 cycles for each wait and 80 for each
// instruction); 473 with boxes of all dims (a box costs the copy engine some 100 cycles, 2 KB or 4); 438 with masks out of the loop;
// 425 with references that leave a sum of 2^20 times the largest probability room: 1.13 PFLOP/s. (All at 1965 MHz. A second of such calls
// in a row draws 950 W, the clock falls to 1.77 GHz, and a call or a replay takes 470.) A quarter, third or half of the exponentials as polynomials took 459, 467, 479: with two warps on a scheduler the instructions
// that this adds cost more than the exponentials that it saves.
// Slots that no row sees: their scores are masked, their values are not fetched but zeroed, so what they hold is never used.
//
// Every wait is on a barrier in shared memory and bounded. A block that gives up goes on without waiting, writes NaN and sets
// error bit 4. Whatever happens, the issuing warp leaves when everything that it has issued is done and every barrier that it
// has committed to has been arrived at, and the fetching warp when its copies are done.

#include "remp_kv_attend.h"
#include "remp_kv_boxes.h"
#include "remp_kvq_device.h"
#include "remp_tensor.h"

namespace remp {

namespace {

constexpr float kUnset = -3e38f;     // reference of a row that has seen nothing
constexpr int kMostSplits = 64;

// References. bfloat16: a row's sum of all its probabilities stays at `bound`, so the 64 parts that its keys may be split into have
// at most 1/2, and sums of p V stay below V's largest number; a new reference puts the largest probability at 2^start, 20 powers
// of two below (about a million tokens that weigh the same move it once), and as p and V have the same exponents, nothing is lost
// on the way for V of 2^-70 and more. Half: its 2^-14 to 2^16 have to hold probabilities, and its largest V times 2^31 of them
// fits 32 bits, so only the sum of a part of a block is bounded; the 96 keys of one at 2^7 fit (at 2^8, equal keys were weighed
// twice in every block: 681 us instead of 419 for the case above).
template <bool BF>
struct Refs {
    static constexpr float bound = BF ? 0x1p-7f : 0x1p14f, start = BF ? -27.f : 7.f, lift = 20.f;
};

template <int D>
struct Prompt {
    static constexpr int kMats = D == 256 ? 1 : 2, kRows = kMats * kRowsM;
    static constexpr int kKeys = D == 256 ? 64 : 128;
    static constexpr int kChunks = kKeys / 32, kFirst = kChunks - 1;  // of 32 keys; those of a block's first part, one makes the second
    static constexpr int kQ = kRowsM * D * 2, kItem = kKeys * D * 2;  // bytes of a matrix, of a block of K or of V
    static constexpr int kEight = 8 * D * 2;                          // bytes of 8 keys: they lie together, 64 dims behind the other
    static constexpr int kPlaces = 5;                                 // of the ring
    static constexpr int kBytes = kMats * kQ + kPlaces * kItem + 1024;
    // columns of the tensor memory: S and P of two matrices, or of two blocks of keys of one matrix, then O of each matrix
    static constexpr int kO = 2 * kKeys, kUsed = kO + kMats * D, kColumns = kUsed <= 256 ? 256 : 512;
    static constexpr int kSoftmaxWarps = 4 * kMats, kThreads = (kSoftmaxWarps + 2) * 32;
    static constexpr int kPartFloats = kRows * (D + 2);
};

struct PromptArgs {
    KvBoxes boxes;
    KvAttendArgs t;
    int32_t row_blocks;        // of a sequence and KV head at most
    int32_t whole, splits;     // units that one thread block does alone; parts of the keys of each unit behind them
    int32_t tries;             // of the wait for the queries
};

template <int D, bool BF>
__global__ void __launch_bounds__(Prompt<D>::kThreads, 1) kv_prompt_kernel(const __grid_constant__ PromptArgs p_) {
    using Z = Prompt<D>;
    using Ref = Refs<BF>;
    constexpr uint32_t kType = BF ? kShapeBfloat : 0;
    constexpr int kSoftmaxWarps = Z::kSoftmaxWarps, kRows = Z::kRows, kKeys = Z::kKeys, kPlaces = Z::kPlaces;
    const KvAttendArgs& a = p_.t;
    extern __shared__ uint8_t smem_[];
    __shared__ __align__(8) uint64_t bars[12 + 2 * kPlaces];
    __shared__ uint32_t tmem_at;
    __shared__ int dead;
    __shared__ int is_last;
    __shared__ __align__(8) uint8_t gone[4][8];  // of a block of keys: tiles that are not there, or that no row sees

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const KvView& v = a.v;
    grid_begin();

    // ---- this block's rows and keys ----
    // row blocks from the last to the first: the last sees the most keys
    const int part_of = (int)blockIdx.x - p_.whole, splits = part_of < 0 ? 1 : p_.splits, split = part_of < 0 ? 0 : part_of % splits;
    int unit = part_of < 0 ? (int)blockIdx.x : p_.whole + part_of / splits;
    const int head = unit % v.kv_heads;
    unit /= v.kv_heads;
    const int seq = unit % v.num_seqs, block = p_.row_blocks - 1 - unit / v.num_seqs;
    const KvqSpan span = kvq_span(v.query_start[seq], v.query_start[seq + 1], v.seq_lens[seq], v.num_tokens, a.room);
    if (kvq_span_bad(span, v.seq_lens[seq]) && block == 0 && tid == 0) kvq_error(v, kErrBadLength);
    const int qs = span.q0, rows_all = span.queries * a.group, row0 = block * kRows;
    if (row0 >= rows_all) return;
    const int rows = min(kRows, rows_all - row0), len = span.len, first_pos = span.first_pos;
    const int low_limit = first_pos + kv_token_of(a.by_group, row0), high_limit = first_pos + kv_token_of(a.by_group, row0 + rows - 1);
    const int end = max(0, min(len, high_limit + 1)), low_from = kvq_first_key(low_limit, a.window), high_from = kvq_first_key(high_limit, a.window);
    // blocks of keys: those of the first tokens, then those of the window; one range where they would meet
    int begin = min(end, low_from) / kKvqTile * kKvqTile, ahead = (min(min(a.first, end), begin) + kKeys - 1) / kKeys;
    if (ahead * kKeys >= begin) begin = ahead = 0;
    const int blocks_all = ahead + (end - begin + kKeys - 1) / kKeys;
    const int b0 = (int)((long long)blocks_all * split / splits), b1 = (int)((long long)blocks_all * (split + 1) / splits);
    const int blocks = b1 - b0;
    const auto key_of = [&](int j) { return b0 + j < ahead ? (b0 + j) * kKeys : begin + (b0 + j - ahead) * kKeys; };  // the first key of block j

    uint8_t* smem = smem_ + ((1024u - ((uint32_t)__cvta_generic_to_shared(smem_) & 1023u)) & 1023u);
    uint8_t *sq = smem, *ring = smem + Z::kMats * Z::kQ;
    // for each matrix: scores, probabilities and products of the halves of a block; queries; places of the ring (block j of K is item 2j, of V item 2j + 1)
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars);
    const uint32_t s_full = bar, p_full = bar + 16, o_half = bar + 32, o_done = bar + 48, p_half = bar + 64, q_full = bar + 80, all_done = bar + 88, full = bar + 96, vacant = full + 8 * kPlaces;
    // Two matrices take turns: while one's products run, P of the other is made. One alone has two buffers of scores instead, those
    // of the next block are there when P of this one is done.
    const int mats = rows > kRowsM ? 2 : 1, buffers = 3 - mats;
    const bool twin = rows <= kRowsM / 2;  // lanes 64 and on take the same rows as lanes 0 and on
    // scores of block j: their place, and of the barriers that go with it; the phase of these. What a barrier had before that
    // phase is done when the scores are there, so no wait for a phase meets the one two before it.
    const auto at_of = [&](int mat, int j) { return mat + (j & buffers - 1); };
    const auto turn_of = [&](int j) { return j >> buffers - 1 & 1; };
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            const int warps = twin ? 2 * ((rows + 31) / 32) : max(1, min(4, (rows - (buffers == 2 ? 0 : i) * kRowsM + 31) / 32));  // those without rows make no P
            bar_init(s_full + 8 * i, 1), bar_init(p_half + 8 * i, warps), bar_init(p_full + 8 * i, warps), bar_init(o_half + 8 * i, 1), bar_init(o_done + 8 * i, 1);
        }
        for (int i = 0; i < kPlaces; ++i) bar_init(full + 8 * i, 1), bar_init(vacant + 8 * i, 1);
        bar_init(q_full, kSoftmaxWarps), bar_init(all_done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead = 0, is_last = 0;
        for (int i = 0; i < 4; ++i) *reinterpret_cast<unsigned long long*>(gone[i]) = 0;
    }
    if (wid == kSoftmaxWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_at)),
                     "n"(Z::kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = tmem_at;

    if (wid < kSoftmaxWarps) {
        // ---- P and the output: one row to a thread ----
        const int mat = wid >> 2;
        const uint32_t lanes = tmem + ((uint32_t)((wid & 3) * 32) << 16), o_at = lanes + Z::kO + mat * D;
        const bool rest = twin && (tid & kRowsM / 2);  // this thread makes what is left of probabilities
        const int mine_of = twin && tid < kRowsM ? tid & kRowsM / 2 - 1 : tid;
        const int row = row0 + min(mine_of, rows - 1), token = kv_token_of(a.by_group, row), q_head = head * a.group + row - token * a.group;
        const bool rows_here = (mine_of & ~31) < rows, gives = rows_here && !rest, real = mine_of < rows && !rest;  // of this warp, of this thread
        const int limit = min(first_pos + token, len - 1), from = kvq_first_key(first_pos + token, a.window);
        // the warp's 32 rows of Q, coalesced
        if (rows_here) {
            constexpr int kPieces = D / 8, kAtOnce = 32 / kPieces;
#pragma unroll 8
            for (int i = 0; i < 32 / kAtOnce; ++i) {
                const int in = wid * 32 + i * kAtOnce + lane / kPieces, piece = lane % kPieces;
                const int r = row0 + min(twin ? in & kRowsM / 2 - 1 : in, rows - 1), tok = kv_token_of(a.by_group, r);
                const uint4 x = *reinterpret_cast<const uint4*>(a.q.data + (int64_t)(qs + tok) * a.q.s_token + (int64_t)(head * a.group + r - tok * a.group) * a.q.s_head + 8 * piece);
                *reinterpret_cast<uint4*>(sq + mat * Z::kQ + (piece / 8) * (kRowsM * 128) + (in & 127) * 128 + (((piece % 8) ^ (in & 7)) << 4)) = x;
            }
        }
        for_tensor_cores();
        __syncwarp();
        if (lane == 0) bar_arrive(q_full);

        // of twins: which part of a probability this thread makes. (Half numbers below 2^-14 have fewer bits than are taken for the first:
        // 2^-22 of a row's largest probability and less.)
        const uint32_t sign = rest ? 0x80000000u : 0u;
        const float keep = rest ? kAndMore : 0.f, least = rest ? kLeastHalf : 0.f;
        float ref = kUnset, sum = 0.f;
#pragma unroll 1
        for (int j = 0; j < (rows_here ? blocks : 0); ++j) {
            const int at = at_of(mat, j);
            const uint32_t s_at = lanes + at * kKeys;
            bar_wait(s_full + 8 * at, turn_of(j), &dead);
            __syncwarp();
            tmem_after();
            const int key0 = key_of(j);
            const unsigned long long missing = *reinterpret_cast<const volatile unsigned long long*>(gone[j & 3]);
            const bool whole = missing == 0 && key0 + kKeys - 1 <= min(low_limit, len - 1) && (key0 >= high_from || key0 + kKeys <= a.first);
            if (!whole) {
                // scores of keys that the row does not see become -infinity where they lie: few blocks have any
#pragma unroll 1
                for (int c = 0; c < Z::kChunks; ++c) {
                    const int last = limit - key0 - 32 * c, least = from - key0 - 32 * c, few = a.first - key0 - 32 * c;
                    uint32_t seen = last >= 31 ? 0xffffffffu : last < 0 ? 0u : (2u << last) - 1;
                    seen &= (least <= 0 ? 0xffffffffu : least >= 32 ? 0u : ~0u << least) | (few >= 32 ? 0xffffffffu : few <= 0 ? 0u : (1u << few) - 1);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (missing >> (8 * (2 * c + i)) & 1) seen &= ~(0xffffu << (16 * i));
                    uint32_t s[32];
                    tmem_ask32(s_at + 32 * c, s);
                    tmem_there32(s);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(seen >> i & 1)) s[i] = 0xff800000u;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t x[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = s[16 * h + i];
                        tmem_store16(s_at + 32 * c + 16 * h, x);
                    }
                }
                tmem_stored();
            }
            // probabilities of a chunk, two to a word, and their sums
            const auto weigh_pair = [&](const uint32_t(&s)[32], int i, float2(&part)[2]) {
                float2 x = fma2(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), make_float2(a.scale_log2, a.scale_log2), make_float2(-ref, -ref));
                x.x = exp2_approx(x.x), x.y = exp2_approx(x.y);
                part[i & 1] = add2(part[i & 1], x);
                return x;
            };
            const auto weigh = [&](const uint32_t(&s)[32], uint32_t* p, float2(&part)[2]) {
                if (!twin) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 x = weigh_pair(s, i, part);
                        p[i] = pack2(x.x, x.y, BF);
                    }
                } else {  // one way for all warps: x * keep + first bits, with (0, +) or (1 + 2^-22, -)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 x = weigh_pair(s, i, part);
                        constexpr uint32_t kBits = BF ? 0xffff0000u : 0xffffe000u;
                        float2 y = make_float2(__uint_as_float((__float_as_uint(x.x) & kBits) ^ sign), __uint_as_float((__float_as_uint(x.y) & kBits) ^ sign));
                        y = fma2(x, make_float2(keep, keep), y);
                        if (!BF) y = make_float2(fmaxf(y.x, fminf(x.x, least)), fmaxf(y.y, fminf(x.y, least)));
                        p[i] = pack2(y.x, y.y, BF);
                    }
                }
            };
            const auto total_of = [](const float2(&part)[2]) {
                const float2 x = add2(part[0], part[1]);
                return x.x + x.y;
            };
            // Rows whose probabilities of chunks [c0, c1) outgrow the bound get another reference; what they have so far falls with it.
            const auto outgrown = [&](float held, int c0, int c1) {
                float top = -INFINITY;
#pragma unroll 1
                for (int c = c0; c < c1; ++c) {
                    uint32_t s[32];
                    tmem_ask32(s_at + 32 * c, s);
                    tmem_there32(s);
#pragma unroll
                    for (int i = 0; i < 32; ++i) top = fmaxf(top, __uint_as_float(s[i]));
                }
                float now = ref;
                if (held > Ref::bound) now = fmaxf(top * a.scale_log2 - Ref::start, BF ? ref + Ref::lift : ref);
                const float fall = exp2_approx(ref - now);
                ref = now, sum *= fall;
                if (j + c0 == 0) return;  // no products yet
                // products so far are done: of the block before, of this one's first part
                if (c0 > 0) bar_wait(o_half + 8 * at, turn_of(j), &dead);
                else bar_wait(o_done + 8 * at_of(mat, j - 1), turn_of(j - 1), &dead);
                __syncwarp();
                tmem_after();
#pragma unroll 1
                for (int i = 0; i < D; i += 16) {
                    uint32_t o[16];
                    tmem_load16(o_at + i, o);
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * fall);
                    tmem_store16(o_at + i, o);
                }
                tmem_stored();
            };
            const auto put = [&](int c, const uint32_t* p) {
                uint32_t x[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = p[i];
                tmem_store16(s_at + 16 * c, x);
            };
            const auto tell = [&](uint32_t b) {
                tmem_stored();
                tmem_before();
                __syncwarp();
                if (lane == 0) bar_arrive(b + 8 * at);
            };
            uint32_t s[2][32], p[16 * Z::kFirst];
#pragma unroll 1
            for (int round = 0;; ++round) {
                float2 part[2] = {};
                tmem_ask32(s_at, s[0]);
                tmem_there32(s[0]);
#pragma unroll
                for (int c = 0; c < Z::kFirst; ++c) {  // the next chunk comes meanwhile
                    tmem_ask32(s_at + 32 * (c + 1), s[c + 1 & 1]);
                    weigh(s[c & 1], p + 16 * c, part);
                    tmem_there32(s[c + 1 & 1]);
                }
                const float total = total_of(part), held = BF ? sum + total : total;
                if (round || !__any_sync(0xffffffffu, held > Ref::bound)) {
                    sum += total;
                    break;
                }
                outgrown(held, 0, Z::kFirst);
            }
#pragma unroll
            for (int c = 0; c < Z::kFirst; ++c) put(c, p + 16 * c);
            tell(p_half);
#pragma unroll 1
            for (int round = 0;; ++round) {
                float2 part[2] = {};
                weigh(s[Z::kFirst & 1], p, part);
                const float total = total_of(part), held = BF ? sum + total : total;
                if (round || !__any_sync(0xffffffffu, held > Ref::bound)) {
                    sum += total;
                    break;
                }
                outgrown(held, Z::kFirst, Z::kChunks);
            }
            put(Z::kFirst, p);
            tell(p_full);
        }
        const bool some = blocks > 0 && rows_here;
        if (some) {
            bar_wait(o_done + 8 * at_of(mat, blocks - 1), turn_of(blocks - 1), &dead);
            __syncwarp();
            tmem_after();
        }
        // O of this thread's row, dims from i on, in steps of 32; of twins the first bits' and the rest's
        float* const rests = reinterpret_cast<float*>(sq) + mine_of;  // [dim][64]; the queries have met all keys
        if (twin && blocks > 0) {
#pragma unroll 1
            for (int i = 0; i < (rows_here && rest ? D : 0); i += 32) {
                uint32_t o[32];
                tmem_load32(o_at + i, o);
#pragma unroll
                for (int k = 0; k < 32; ++k) rests[(i + k) * (kRowsM / 2)] = __uint_as_float(o[k]);
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
        }
        const auto load_o = [&](int i, uint32_t(&o)[32]) {
            if (some) {
                tmem_load32(o_at + i, o);
                if (twin)
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) + rests[(i + k) * (kRowsM / 2)]);
            } else {
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = 0;
            }
        };
        // Whoever gave up said so before its next arrival, and outputs are behind all arrivals: none that went wrong gets here
        // without the mark.
        if (*static_cast<volatile int*>(&dead)) sum = __uint_as_float(0x7fc00000u);
        uint16_t* dst = a.out.data + (int64_t)(qs + token) * a.out.s_token + (int64_t)q_head * a.out.s_head;
        if (splits == 1) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll 1
            for (int i = 0; i < (gives ? D : 0); i += 32) {
                uint32_t o[32];
                load_o(i, o);
                if (real)
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) w[x] = pack2(__uint_as_float(o[k + 2 * x]) * inv, __uint_as_float(o[k + 2 * x + 1]) * inv, BF);
                        *reinterpret_cast<uint4*>(dst + i + k) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
            }
            if (real && a.lse) a.lse[(int64_t)(qs + token) * a.q_heads + q_head] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
        } else {
            // a part: [dim][row], then references and sums; the block that comes last adds the parts up in their order
            float* slots = reinterpret_cast<float*>(a.workspace + kAttendCounterBytes);
            float* mine = slots + (int64_t)part_of * Z::kPartFloats;
#pragma unroll 1
            for (int i = 0; i < (gives ? D : 0); i += 32) {
                uint32_t o[32];
                load_o(i, o);
#pragma unroll
                for (int k = 0; k < 32; ++k) mine[(i + k) * kRows + tid] = __uint_as_float(o[k]);
            }
            mine[D * kRows + tid] = ref, mine[(D + 1) * kRows + tid] = sum;
            asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
            if (tid == 0) {
                uint32_t* counter = reinterpret_cast<uint32_t*>(a.workspace) + part_of / splits;
                uint32_t before;
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
                is_last = before == (uint32_t)splits - 1;
                if (is_last) *counter = 0;  // ready for the next call
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
            if (is_last) {
                // 32 rows and 16 dims to a warp at a time, in steps of eight parts' references and four parts' values
                const float* part = slots + (int64_t)(part_of - split) * Z::kPartFloats;
#pragma unroll 1
                for (int task = wid; task < (rows + 31) / 32 * (D / 16); task += kSoftmaxWarps) {
                    const int r = task / (D / 16) * 32 + lane, d = task % (D / 16) * 16;
                    const int my_row = row0 + min(r, rows - 1), my_token = kv_token_of(a.by_group, my_row), my_head = head * a.group + my_row - my_token * a.group;
                    const float* refs = part + D * kRows + r;
                    float top = kUnset, all = 0.f, o[16];
#pragma unroll 8
                    for (int i = 0; i < splits; ++i) top = fmaxf(top, __ldcg(refs + (int64_t)i * Z::kPartFloats));
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] = 0.f;
#pragma unroll 4
                    for (int i = 0; i < splits; ++i) {
                        const float* x = part + (int64_t)i * Z::kPartFloats + d * kRows + r;
                        const float f = exp2_approx(__ldcg(refs + (int64_t)i * Z::kPartFloats) - top);
                        all = fmaf(f, __ldcg(refs + (int64_t)i * Z::kPartFloats + kRows), all);
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = fmaf(f, __ldcg(x + k * kRows), o[k]);
                    }
                    const float inv = all == 0.f ? 0.f : 1.f / all;
                    if (r < rows) {
                        uint16_t* to = a.out.data + (int64_t)(qs + my_token) * a.out.s_token + (int64_t)my_head * a.out.s_head + d;
                        uint32_t w[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) w[x] = pack2(o[2 * x] * inv, o[2 * x + 1] * inv, BF);
                        *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4*>(to + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                        if (a.lse && d == 0)
                            a.lse[(int64_t)(qs + my_token) * a.q_heads + my_head] = all == 0.f ? -INFINITY : (top + log2f(all)) * 0.69314718055994531f;
                    }
                }
            }
        }
    } else if (wid == kSoftmaxWarps) {
        // ---- matrix instructions: one thread waits and issues ----
        if (elect_one()) {
            const int n = blocks, live = mats;
            const uint64_t q_at = operand_at((uint32_t)__cvta_generic_to_shared(sq)), ring_at = operand_at((uint32_t)__cvta_generic_to_shared(ring));
            // K and V: from 8 keys to the next 8; V, across the keys: from 64 dims to the next 64
            constexpr uint64_t kOfK = keys_apart(Z::kEight), kOfV = kOfK + ((uint64_t)((1024 >> 4) - 1) << 16);
            const auto scores = [&](int j, int mat, uint64_t k_block) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_smem_one(tmem + at_of(mat, j) * kKeys, q_at + (mat * Z::kQ + (k / 4) * (kRowsM * 128) + (k % 4) * 32 >> 4),
                                               k_block + ((k / 4) * 1024 + (k % 4) * 32 >> 4), kShape<kKeys> | kType, k > 0);
                commit_one(s_full + 8 * at_of(mat, j));
            };
            // places of the ring that the next block of K, of V has
            int place_v = 1 % kPlaces, place_k = 0;
            uint32_t turn_v = 0, turn_k = 0;
            const auto next_k = [&] {
                if ((place_k += 2) >= kPlaces) place_k -= kPlaces, turn_k ^= 1;
            };
            const auto scores_alone = [&](int j) {  // of every matrix, behind what was issued
                bar_wait(full + 8 * place_k, turn_k, &dead);
                tmem_after();
#pragma unroll 1
                for (int mat = 0; mat < live; ++mat) scores(j, mat, ring_at + (uint32_t)(place_k * (Z::kItem >> 4)) + kOfK);
                commit_one(vacant + 8 * place_k);
                next_k();
            };
            if (n > 0) {
                bar_wait(q_full, 0, &dead, p_.tries);
                scores_alone(0);
            }
#pragma unroll 1
            for (int j = 0; j < n; ++j) {
                // P.V of block j and the scores of the next. Of one matrix these come first and take the other buffer, whose
                // products were issued a block ago; of two they follow, matrix by matrix, and take the place of the probabilities
                // before them: instructions run in the order of issue.
                if (buffers == 2 && j + 1 < n) scores_alone(j + 1);
                const uint64_t v_block = ring_at + (uint32_t)(place_v * (Z::kItem >> 4)) + kOfV, k_block = ring_at + (uint32_t)(place_k * (Z::kItem >> 4)) + kOfK;
                const bool more = buffers == 1 && j + 1 < n;
                bar_wait(full + 8 * place_v, turn_v, &dead);
#pragma unroll 1
                for (int mat = 0; mat < live; ++mat) {
                    const int at = at_of(mat, j);
                    const uint32_t o_at = tmem + Z::kO + mat * D, p_at = tmem + at * kKeys;
                    bar_wait(p_half + 8 * at, turn_of(j), &dead);
                    tmem_after();
#pragma unroll
                    for (int k = 0; k < 2 * Z::kFirst; ++k) mma_tmem_one<D, kType | kShapeBAcross>(o_at, p_at + 8 * k, v_block + (2 * k * Z::kEight >> 4), k ? 1 : j);
                    commit_one(o_half + 8 * at);
                    bar_wait(p_full + 8 * at, turn_of(j), &dead);
                    tmem_after();
#pragma unroll
                    for (int k = 2 * Z::kFirst; k < kKeys / 16; ++k) mma_tmem_one<D, kType | kShapeBAcross>(o_at, p_at + 8 * k, v_block + (2 * k * Z::kEight >> 4), 1);
                    commit_one(o_done + 8 * at);
                    if (more) {
                        if (mat == 0) bar_wait(full + 8 * place_k, turn_k, &dead);
                        scores(j + 1, mat, k_block);
                    }
                }
                commit_one(vacant + 8 * place_v);
                if (more) {
                    commit_one(vacant + 8 * place_k);
                    next_k();
                }
                if ((place_v += 2) >= kPlaces) place_v -= kPlaces, turn_v ^= 1;
            }
            // Nothing stays in flight, whatever happened: a barrier of its own stands behind everything, since a block that gave up may
            // have run ahead of the others by several phases. Then the last arrival on each of these.
            commit_one(all_done);
            bar_drain(all_done, 1, &dead);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int times = buffers == 2 ? (n + 1 - i) / 2 : n;
                bar_drain(s_full + 8 * i, times, &dead), bar_drain(o_half + 8 * i, times, &dead), bar_drain(o_done + 8 * i, times, &dead);
            }
#pragma unroll
            for (int i = 0; i < kPlaces; ++i) bar_drain(vacant + 8 * i, (2 * n - i + kPlaces - 1) / kPlaces, &dead);
        }
        __syncwarp();
    } else {
        // ---- keys and values: a tile of 16 tokens to a lane, in boxes; of V those with slots that no row sees by rows, with zeros there ----
        constexpr int kTiles = kKeys / kKvqTile, kTile = 2 * Z::kEight;
        const int32_t* row = v.tables + (int64_t)seq * v.max_blocks;
        const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
        // Whether a row sees something of the tile from `key` on; others are not looked up: their pages may have been given back.
        const auto wanted = [&](int key) { return lane < kTiles && key < end && (key + kKvqTile > low_from || key < a.first); };
        // This lane's tile of block j: its block (-1: not there) and first token in it. Asked for a block ahead.
        const auto find = [&](int j) {
            int2 r = make_int2(-1, 0);
            const int key = key_of(j) + lane * kKvqTile;
            if (j < blocks && wanted(key)) {
                const int tile = key / kKvqTile, in_row = tile / v.block_tiles;
                r = make_int2(__ldg(row + in_row), (tile - in_row * v.block_tiles) * kKvqTile);
            }
            return r;
        };
        int2 at = make_int2(-1, 0), next = find(0);
        int items = 0;
#pragma unroll 1
        for (; items < 2 * blocks; ++items) {
            const int j = items >> 1, place = items % kPlaces, turn = items / kPlaces;
            const bool of_v = items & 1;
            const int key0 = key_of(j), key = key0 + lane * kKvqTile;
            if (!of_v) {
                at = next, next = find(j + 1);
                if ((uint32_t)at.x >= (uint32_t)v.nb) {
                    if (wanted(key)) kvq_error(v, kErrBadBlock);
                    at.x = -1;
                }
            }
            if (turn > 0) bar_wait(vacant + 8 * place, (turn - 1) & 1, &dead);
            if (__any_sync(0xffffffffu, *static_cast<volatile int*>(&dead))) break;  // what is asked for is waited for below
            if (!of_v && lane < kTiles) gone[j & 3][lane] = at.x < 0;
            // What unseen slots of K hold is masked score by score; of V they would meet probabilities of 0, so there they are zeros.
            const bool every = at.x >= 0 && (!of_v || (key + kKvqTile <= end && (key >= low_from || key + kKvqTile <= a.first)));
            const uint32_t boxes = __ballot_sync(0xffffffffu, every);
            const uint32_t dst = ring_at + place * Z::kItem;
            for (uint32_t others = of_v ? ~boxes & ((1u << kTiles) - 1) : 0; others; others &= others - 1) {
                const int t = __ffs(others) - 1, id = __shfl_sync(0xffffffffu, at.x, t), token = __shfl_sync(0xffffffffu, at.y, t), first_key = key0 + t * kKvqTile;
                const uint8_t* src = v.base + (int64_t)id * v.s_block + v.s_kv + (int64_t)head * v.s_head + (int64_t)token * v.s_token;
                uint4 x[kKvqTile * (D / 8) / 32];
#pragma unroll
                for (int i = 0; i < kKvqTile * (D / 8) / 32; ++i) {
                    const int r = (i * 32 + lane) / (D / 8), piece = (i * 32 + lane) % (D / 8);
                    const bool real = id >= 0 && first_key + r < end && (first_key + r >= low_from || first_key + r < a.first);
                    x[i] = real ? *reinterpret_cast<const uint4*>(src + r * v.s_token + piece * 16) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < kKvqTile * (D / 8) / 32; ++i) {
                    const int r = (i * 32 + lane) / (D / 8), piece = (i * 32 + lane) % (D / 8);
                    *reinterpret_cast<uint4*>(ring + place * Z::kItem + t * kTile + (r / 8) * Z::kEight + (piece / 8) * 1024 + (r & 7) * 128 + (((piece % 8) ^ (r & 7)) << 4)) = x[i];
                }
            }
            for_tensor_cores();
            __syncwarp();
            if (lane == 0) bar_arrive_expecting(full + 8 * place, __popc(boxes) * (kKvqTile * D * 2));
            __syncwarp();
            if (every) bring_tile(dst + lane * kTile, of_v ? &p_.boxes.v : &p_.boxes.k, full + 8 * place, at.y / 8, at.x * p_.boxes.i_block + head * p_.boxes.i_head);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kPlaces; ++i) bar_drain(full + 8 * i, max(0, items - i + kPlaces - 1) / kPlaces, &dead);
        __syncwarp();
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    __syncwarp();
    if (wid == kSoftmaxWarps)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Z::kColumns));
    if (tid == 0 && dead) kvq_error(v, kErrWaitLimit);
}

template <int D>
cudaError_t launch(PromptArgs& p, bool bf, int sms, int max_rows, cudaStream_t stream) {
    using Z = Prompt<D>;
    static_assert(Z::kBytes + 512 <= 227 * 1024, "shared memory");
    const KvView& v = p.t.v;
    p.row_blocks = (max_rows + Z::kRows - 1) / Z::kRows;
    const int64_t units = (int64_t)p.row_blocks * v.num_seqs * v.kv_heads;
    // a unit is a thread block's work; those that are left when the others have filled the GPU whole times share it, each
    // one's keys split
    constexpr int kParts = (int)((kAttendWorkspace - kAttendCounterBytes) / (Z::kPartFloats * 4));
    const int places = std::min(sms, kParts);
    const int64_t rest = units % sms;
    p.splits = rest ? (int)std::min<int64_t>(kMostSplits, places / rest) : 1;
    if (p.splits < 2) p.splits = 1;
    p.whole = (int)(p.splits > 1 ? units - rest : units);
    static_assert(kParts >= 148 && kParts <= 2 * kAttendMaxCtas, "workspace");  // splits of two at least: a counter for two parts
    if (units > 0x7fffffff / kMostSplits) return cudaErrorInvalidConfiguration;
    p.tries = prompt_wait_tries();
    return launch_after(bf ? kv_prompt_kernel<D, true> : kv_prompt_kernel<D, false>, p.whole + (units - p.whole) * p.splits, Z::kThreads, Z::kBytes, stream, p);
}

}  // namespace

cudaError_t launch_kv_prompt(const KvAttendArgs& a, int32_t head_dim, bool bf, int sms, int32_t max_rows, cudaStream_t stream) {
    PromptArgs p{};
    p.t = a, p.splits = 1;
    if (cudaError_t e = kv_boxes(a.v, head_dim, bf, &p.boxes)) return e;
    return head_dim == 64 ? launch<64>(p, bf, sms, max_rows, stream)
           : head_dim == 128 ? launch<128>(p, bf, sms, max_rows, stream) : launch<256>(p, bf, sms, max_rows, stream);
}

}  // namespace remp
