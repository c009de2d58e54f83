// Attention over the 4-bit cache for many queries per sequence (prompts and their chunks), on the tensor cores' own memory.
//
// Mathematics: softmax(scale * q.K^T + mask).V, one thread block for 256 rows (tokens x query heads of one KV head; two
// matrices of 128) and a range of the keys, block by block of kKeys keys: S = Q.K^T, P = 2^(S*back - ref), O += P.V, with a
// running reference for each row that moves only when the probabilities of 32 keys outgrow kBound.
// Rounding: q is exact in half after a power of two per row; keys and values s*c + m are rounded to half and so is P (twice
// where a reference moves in the middle of its block of keys); S, O, sums and references are in 32 bits.
// Range: halves hold K/4 and 8 V where every token of a thread block's keys has its largest step or minimum in a range that allows
// it (2^-7 to 2^13, 2^-12 to 2^8). Where one has not, each token gets a power of two of its own, which brings that to [2^10,
// 2^11), so that a value is rounded to 11 bits down to 2^-24 of the token's largest. S is multiplied with K's powers; V's go
// into P, and the reference bounds P with them in it, so a row that sees only tokens of small values is as exact as any
// other. The sums of P are without them. The warps that make no P look at all the parameters first, while the queries come.
//
// Bound: tensor cores (4*D flops for each row and key), then issue slots and exponentials: eight warps turn codes into halves
// once for both matrices, eight compute P (a row to a thread), one thread issues the matrix instructions, which run for
// one matrix while P of the other is made. Q, two blocks of K and two of V^T lie in shared memory in rows of 128 bytes,
// 16-byte pieces exchanged within 8 rows (piece ^ (row & 7)); K's codes are stored so that a word gives neighbouring dims
// and V's words of two tokens give a pair of keys, so each 4-byte store of a warp meets 32 different banks. S and P share
// their columns of the tensor memory, O has its own. With 256 dims O takes so much of it that one matrix of 128 rows and
// blocks of 64 keys are left.
//
// Measured: 2 x 2048 queries of 32 heads over 8191 tokens of 4 KV heads, 481 GFLOP, 568 to 594 us in different
// runs: 810 to 847 TFLOP/s, 50 to 52 % of a library product in bf16. Bound by the chain of one matrix, scores to P to products to
// the next scores: some 4750 cycles for a block, 2700 of them from reading S to the last of P. Blocks of 64 keys with two S each,
// which break the chain, took 779 us (both timed with clock reads in the kernel). Looking at the parameters first takes 1 to 4 %
// (8 x 8 units of 40 rows over 4000 keys 51.4 us without, 52.4 with); marks for each tile inside the loops took up to 24 % (2 x
// 1024 queries of 256 dims 562 to 695 us). With powers of their own the call above takes 0.79 ms.
//
// Every wait is on a barrier in shared memory and bounded. A block that gives up goes on without waiting, writes NaN and sets
// error bit 4. Whatever happens, the issuing warp leaves when everything that it has issued is done and every barrier that it
// has committed to has been arrived at, so nothing runs on in freed memory. (Looking before each issue whether the block has
// given up cost calls of few rows a third: the units above 49 to 66 us.)

#include <atomic>
#include <type_traits>

#include "remp_kvq_device.h"
#include "remp_tensor.h"

namespace remp {

namespace {

constexpr float kUnset = -3e38f;     // reference of a row that has seen nothing
constexpr float kBound = 16384.f;    // of the sum of 32 probabilities
constexpr float kStart = 8.f;        // log2 of the largest probability when a reference is set
// What K and V are multiplied with to become halves, as powers of two, where all tokens allow it: the larger of step and
// minimum is from 2^least_of to below 2^most_of. Below, steps lose bits as halves, above, 16 times as much is no half.
// Keys are wide (biases, outliers), values small: K from 2^-7 to 2^13, V from 2^-12 to 2^8.
constexpr int kUpK = -2, kUpV = 3;
__host__ __device__ constexpr int least_of(int up) { return -9 - up; }
__host__ __device__ constexpr int most_of(int up) { return 11 - up; }
constexpr int kMostSplits = 16;
std::atomic<int32_t> g_wait_tries{kWaitTries};  // remp_kvq_set_wait_limit

template <int D>
struct Prompt {
    static constexpr int kMats = D == 256 ? 1 : 2, kRows = kMats * kRowsM;
    static constexpr int kKeys = D == 256 ? 64 : 128, kUnpackWarps = kKeys / kKvqTile;  // a tile to a warp
    static constexpr int kQ = kRowsM * D * 2, kK = kKeys * D * 2, kV = kKeys * D * 2;  // bytes of a matrix, of a block
    static constexpr int kPowers = 4 * 2 * kKeys * 4;  // of K and V, four blocks of keys
    static constexpr int kBytes = kMats * kQ + 2 * (kK + kV) + kPowers + 1024;
    // columns of the tensor memory: S and P of each matrix, then O of each
    static constexpr int kO = kMats * kKeys, kUsed = kO + kMats * D, kColumns = kUsed <= 256 ? 256 : 512;
    static constexpr int kSoftmaxWarps = 4 * kMats, kThreads = (kSoftmaxWarps + kUnpackWarps + 1) * 32;
    static constexpr int kPartFloats = kRows * (D + 2);
};

// ---- codes to halves ----

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t as_word(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }

// Two numbers as halves, kept finite (NaN stays).
__device__ __forceinline__ __half2 finite_halves(float lo, float hi) {
    uint32_t x;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(hi), "f"(lo));
    return as_half2(x);
}
// codes at bits 0..3 of both halves of x, times step, plus low
__device__ __forceinline__ uint32_t halves_of(uint32_t x, __half2 step, __half2 low) {
    uint32_t y;  // 1024 + code: one instruction takes the bits and sets the others
    asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(y) : "r"(x), "r"(0x64006400u));
    return as_word(__hfma2(__hsub2(as_half2(y), __half2half2(__ushort_as_half(0x6400))), step, low));
}
// the four codes of either half of w
__device__ __forceinline__ void four_halves(uint32_t w, __half2 step, __half2 low, uint32_t (&z)[4]) {
    z[0] = halves_of(w, step, low), z[1] = halves_of(w >> 4, step, low), z[2] = halves_of(w >> 8, step, low), z[3] = halves_of(w >> 12, step, low);
}

struct PromptArgs {
    KvqView v;
    KvqRows q, out;
    float* lse;
    uint8_t* workspace;
    float scale_log2;
    int32_t group, q_heads, window, room;
    uint32_t by_group;
    int32_t row_blocks;        // of a sequence and KV head at most
    int32_t whole, splits;     // units that one thread block does alone; parts of the keys of each unit behind them
    int32_t tries;             // of the wait for the queries
};

__device__ __forceinline__ int prompt_token(const PromptArgs& a, int row) { return a.by_group ? (int)__umulhi((uint32_t)row, a.by_group) : row; }

template <int D>
struct RawK { uint32_t w[2][D / 32], par[2][D / 64]; };  // tokens g, g + 8: a lane's words and the parameters
template <int D>
struct RawV { uint32_t w[4][D / 64], par[4][D / 64]; };  // tokens 2t, 2t + 1, 2t + 8, 2t + 9

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
    if constexpr (N == 1) {
        w[0] = __ldcg(reinterpret_cast<const uint32_t*>(p));
    } else if constexpr (N == 2) {
        const uint2 x = __ldcg(reinterpret_cast<const uint2*>(p));
        w[0] = x.x, w[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 x = __ldcg(reinterpret_cast<const uint4*>(p + 4 * i));
            w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
        }
    }
}

// A lane's words of a tile of K, or of V; `tile` null: nothing is there.
template <int D>
__device__ __forceinline__ void load_k(const uint8_t* tile, int g, int t, RawK<D>& r) {
    if (tile) {
        const uint8_t *codes = tile + g * (D / 2) + t * (D / 8), *params = tile + kKvqTile * D / 2 + g * (D / 16);
#pragma unroll
        for (int h = 0; h < 2; ++h) load_words(codes + h * 4 * D, r.w[h]), load_words(params + h * (D / 2), r.par[h]);
    }
}
// The tokens from `valid` on are not there: their values are 0, whatever their slots hold.
template <int D>
__device__ __forceinline__ void load_v(const uint8_t* tile, int valid, int g, int t, RawV<D>& r) {
    if (tile) {
        const uint8_t *codes = tile + t * D + g * (D / 16), *params = tile + kKvqTile * D / 2 + t * (D / 8);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            load_words(codes + (j >> 1) * 4 * D + (j & 1) * (D / 2), r.w[j]), load_words(params + (j >> 1) * (D / 2) + (j & 1) * (D / 16), r.par[j]);
    }
    if (!tile || valid < kKvqTile) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!tile || 2 * t + (j & 1) + (j >> 1) * 8 >= valid)
#pragma unroll
                for (int i = 0; i < D / 64; ++i) r.par[j][i] = 0;
    }
}

// The larger of step and minimum of a token's groups, as bits of a bfloat16: a value is at most 16 times as large.
template <int G>
__device__ __forceinline__ uint32_t largest_of(const uint32_t (&par)[G]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < G; ++i) most = __vmaxu2(most, par[i] & 0x7fff7fffu);
    return max(most >> 16, most & 0xffffu);
}
__device__ __forceinline__ bool out_of_range(int up, uint32_t largest) {
    const uint32_t least = (uint32_t)(127 + least_of(up)) << 7, most = (uint32_t)(127 + most_of(up)) << 7;  // as bits of bfloat16
    return largest != 0 && largest - least >= most - least;
}
// A token's power of two, over that of all tokens. Groups of NaN and infinity do not count. Of V 2^-78 to 2^103, so that sums
// of P without the powers stay inside 32 bits' range; of K 2^-114 to 2^110.
template <int UP, int G>
__device__ __forceinline__ float power_of(const uint32_t (&par)[G]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < G; ++i)
        if ((par[i] & 0x7f800000u) != 0x7f800000u) most = max(most, max((par[i] & 0x7fffffffu) >> 16, par[i] & 0x7fffu));
    return most ? __uint_as_float((uint32_t)(127 + UP + max(UP == kUpV ? -81 : -112, min(UP == kUpV ? 100 : 112, (int)(most >> 7) - 127 - 10))) << 23) : 1.f;
}
__host__ __device__ constexpr float two_to(int e) { return e < 0 ? 1.f / (float)(1 << -e) : (float)(1 << e); }
// What steps and minima are multiplied with: 2^UP / power.
template <int UP>
__device__ __forceinline__ float down_of(float power) { return __uint_as_float(((uint32_t)(254 + UP) << 23) - __float_as_uint(power)); }

// Rows of K, a key each: place[c] is where piece c of this lane's 8 keys' rows begins, for its words of the pieces.
template <int D>
__device__ __forceinline__ void store_k(uint8_t* const (&place)[8], const RawK<D>& r, const float (&down)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int grp = 0; grp < D / 64; ++grp) {
            const float s = bf_low(r.par[h][grp]) * down[h], m = bf_high(r.par[h][grp]) * down[h];
            const __half2 step = finite_halves(s, s), low = finite_halves(m, m);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint32_t z[4];
                four_halves(r.w[h][2 * grp + x], step, low, z);
#pragma unroll
                for (int b = 0; b < 4; ++b) *reinterpret_cast<uint32_t*>(place[4 * x + b] + (8 * h + grp * Prompt<D>::kKeys) * 128) = z[b];
            }
        }
}

// Rows of V^T, a dim each: row 8n + g from `place` on, two keys to a word.
template <int D>
__device__ __forceinline__ void store_v(uint8_t* const (&place)[2], const RawV<D>& r, const float (&down)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int grp = 0; grp < D / 64; ++grp) {
            const uint32_t p0 = r.par[2 * h][grp], p1 = r.par[2 * h + 1][grp];
            const float d0 = down[2 * h], d1 = down[2 * h + 1];
            const __half2 step = finite_halves(bf_low(p0) * d0, bf_low(p1) * d1), low = finite_halves(bf_high(p0) * d0, bf_high(p1) * d1);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint32_t z[4];
                four_halves(__byte_perm(r.w[2 * h][grp], r.w[2 * h + 1][grp], x ? 0x7632 : 0x5410), step, low, z);
#pragma unroll
                for (int b = 0; b < 4; ++b) *reinterpret_cast<uint32_t*>(place[h] + (grp * 64 + 8 * (4 * x + b)) * 128) = z[b];
            }
        }
}

template <int D, bool BF>
__global__ void __launch_bounds__(Prompt<D>::kThreads, 1) kvq_prompt_kernel(const __grid_constant__ PromptArgs a) {
    using Z = Prompt<D>;
    extern __shared__ uint8_t smem_[];
    __shared__ __align__(8) uint64_t bars[16];
    __shared__ uint32_t tmem_at;
    __shared__ int dead;
    __shared__ int is_last;
    __shared__ int own_powers;  // tokens have powers of two of their own
    constexpr int kSoftmaxWarps = Z::kSoftmaxWarps, kUnpackWarps = Z::kUnpackWarps, kRows = Z::kRows;
    __shared__ __align__(8) uint8_t gone[4][8];  // of a block of keys: tiles that are not there

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const KvqView& v = a.v;
    grid_begin();

    // ---- this block's rows and keys ----
    // row blocks from the last to the first: the last sees the most keys
    const int part_of = (int)blockIdx.x - a.whole, splits = part_of < 0 ? 1 : a.splits, split = part_of < 0 ? 0 : part_of % splits;
    int unit = part_of < 0 ? (int)blockIdx.x : a.whole + part_of / splits;
    const int head = unit % v.kv_heads;
    unit /= v.kv_heads;
    const int seq = unit % v.num_seqs, block = a.row_blocks - 1 - unit / v.num_seqs;
    const KvqSpan span = kvq_span(v.query_start[seq], v.query_start[seq + 1], v.seq_lens[seq], v.num_tokens, a.room);
    const int qs = span.q0, rows_all = span.queries * a.group, row0 = block * kRows;
    if (row0 >= rows_all) return;
    const int rows = min(kRows, rows_all - row0), len = span.len, first_pos = span.first_pos;
    if (kvq_span_bad(span, v.seq_lens[seq]) && tid == 0) kvq_error(v, kErrBadLength);
    const int low_limit = first_pos + prompt_token(a, row0), high_limit = first_pos + prompt_token(a, row0 + rows - 1);
    const int end = max(0, min(len, high_limit + 1)), begin = min(end, kvq_first_key(low_limit, a.window)) / kKvqTile * kKvqTile;
    const int blocks_all = (end - begin + Z::kKeys - 1) / Z::kKeys;
    const int b0 = (int)((long long)blocks_all * split / splits), b1 = (int)((long long)blocks_all * (split + 1) / splits);
    const int blocks = b1 - b0, first_key = begin + b0 * Z::kKeys;

    uint8_t* smem = smem_ + ((1024u - ((uint32_t)__cvta_generic_to_shared(smem_) & 1023u)) & 1023u);
    uint8_t *sq = smem, *sk = smem + Z::kMats * Z::kQ, *sv = sk + 2 * Z::kK;
    float* const powers = reinterpret_cast<float*>(sv + 2 * Z::kV);  // [block & 3][K, V][key]
    // blocks of K and V come and go (two places each); scores, probabilities and outputs of each matrix; queries
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars);
    const uint32_t k_full = bar, k_free = bar + 16, v_full = bar + 32, v_free = bar + 48, s_full = bar + 64, p_full = bar + 80, o_done = bar + 96, q_full = bar + 112, all_done = bar + 120;
    const int mats = rows > kRowsM ? 2 : 1;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            bar_init(k_full + 8 * i, kUnpackWarps), bar_init(v_full + 8 * i, kUnpackWarps), bar_init(k_free + 8 * i, 1), bar_init(v_free + 8 * i, 1);
            bar_init(s_full + 8 * i, 1), bar_init(p_full + 8 * i, 4), bar_init(o_done + 8 * i, 1);
        }
        bar_init(q_full, kSoftmaxWarps), bar_init(all_done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead = 0, is_last = 0, own_powers = 0;
        for (int i = 0; i < 4; ++i) *reinterpret_cast<unsigned long long*>(gone[i]) = 0;
    }
    if (wid == kSoftmaxWarps + kUnpackWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_at)),
                     "n"(Z::kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = tmem_at;

    // Does a token need a power of its own? The warps that make no P look, at tiles nth, nth + kLookers and so on, 16 bytes of
    // parameters to a lane, while the others bring the queries; all meet behind it.
    constexpr int kLookers = kUnpackWarps + 1;
    const auto look = [&](int nth) {
        constexpr int kLanes = D / 16, kTiles = 16 / kLanes, kAhead = D == 256 ? 16 : 4;  // lanes of a tile's K or V, tiles of a load, loads ahead
        const int tiles = (max(0, min(end, first_key + blocks * Z::kKeys) - first_key) + kKvqTile - 1) / kKvqTile;
        const bool of_v = lane / kLanes & 1;
        const int sub = lane / (2 * kLanes), first_token = lane % kLanes * (256 / D);
        const uint8_t* params = v.base + (int64_t)head * v.s_head + (of_v ? v.s_kv : 0) + kKvqTile * D / 2 + lane % kLanes * 16;
        bool odd = false;
#pragma unroll 1
        for (int t0 = nth; t0 < tiles; t0 += kLookers * 32) {
            const int mine = t0 + lane * kLookers, tile = first_key / kKvqTile + mine;  // where this lane's tile is in the pool
            long long at = -1;
            if (mine < tiles) {
                const int in_row = tile / v.block_tiles, id = __ldcg(v.tables + (int64_t)seq * v.max_blocks + in_row);
                if ((uint32_t)id < (uint32_t)v.nb) at = (int64_t)id * v.s_block + (tile - in_row * v.block_tiles) * (kKvqTile * kvq_token_bytes(D));
            }
#pragma unroll 1
            for (int i = 0; i < 32 && t0 + i * kLookers < tiles; i += kAhead * kTiles) {
                uint4 par[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const long long from = __shfl_sync(0xffffffffu, at, i + k * kTiles + sub);
                    par[k] = from >= 0 ? __ldcg(reinterpret_cast<const uint4*>(params + from)) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const uint32_t w[4] = {par[k].x, par[k].y, par[k].z, par[k].w};
                    const int token = first_key + (t0 + (i + k * kTiles + sub) * kLookers) * kKvqTile + first_token;
#pragma unroll
                    for (int u = 0; u < 256 / D; ++u) {
                        uint32_t one[D / 64];
#pragma unroll
                        for (int x = 0; x < D / 64; ++x) one[x] = w[u * (D / 64) + x];
                        odd |= token + u < len && out_of_range(of_v ? kUpV : kUpK, largest_of(one));
                    }
                }
            }
        }
        if (__any_sync(0xffffffffu, odd) && lane == 0) *static_cast<volatile int*>(&own_powers) = 1;
    };
    const auto all_meet = [&] {
        asm volatile("bar.sync 2, %0;" ::"n"(Z::kThreads) : "memory");
        return *static_cast<volatile int*>(&own_powers) != 0;
    };

    if (wid < kSoftmaxWarps) {
        // ---- P and the output: one row to a thread ----
        const int mat = wid >> 2;
        const uint32_t lanes = tmem + ((uint32_t)((wid & 3) * 32) << 16), s_at = lanes + mat * Z::kKeys, o_at = lanes + Z::kO + mat * D;
        const int row = row0 + min(tid, rows - 1), token = prompt_token(a, row), q_head = head * a.group + row - token * a.group;
        const bool real = tid < rows;
        const int limit = min(first_pos + token, len - 1), from = kvq_first_key(first_pos + token, a.window);
        float back;
        {
            const uint16_t* src = a.q.data + (int64_t)(qs + token) * a.q.s_token + (int64_t)q_head * a.q.s_head;
            uint32_t most = 0;
#pragma unroll 4
            for (int i = 0; i < D / 8; ++i) {
                const uint4 x = reinterpret_cast<const uint4*>(src)[i];
                most = __vmaxu2(most, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
            }
            most = max(most >> 16, most & 0xffffu);
            const float top = BF ? __uint_as_float(most << 16) : __half2float(__ushort_as_half((unsigned short)most));
            const int e = most ? max(-120, min(110, 3 - ((int)(__float_as_uint(top) >> 23) - 127))) : 0;
            const float up = __uint_as_float((uint32_t)(127 + e) << 23);
            back = fmaxf(a.scale_log2 * two_to(-kUpK) * __uint_as_float((uint32_t)(127 - e) << 23), 1.2e-38f);
#pragma unroll 4
            for (int i = 0; i < D / 8; ++i) {
                const uint4 x = reinterpret_cast<const uint4*>(src)[i];
                uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 f = BF ? make_float2(bf_low(w[k]), bf_high(w[k])) : __half22float2(as_half2(w[k]));
                    w[k] = pack2(f.x * up, f.y * up, false);
                }
                *reinterpret_cast<uint4*>(sq + mat * Z::kQ + (i / 8) * (kRowsM * 128) + (tid & 127) * 128 + (((i % 8) ^ (tid & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            for_tensor_cores();
            __syncwarp();
            if (lane == 0) bar_arrive(q_full);
        }
        const bool odd = all_meet();
        float ref = kUnset, sum = 0.f;
        const auto make_p = [&](auto own) {
            constexpr bool kOwn = decltype(own)::value;
#pragma unroll 1
            for (int j = 0; j < (mat < mats ? blocks : 0); ++j) {
                bar_wait(s_full + 8 * mat, j & 1, &dead);
                __syncwarp();
                tmem_after();
                const int key0 = first_key + j * Z::kKeys;
                const unsigned long long missing = *reinterpret_cast<const volatile unsigned long long*>(gone[j & 3]);
                const bool whole = missing == 0 && key0 + Z::kKeys - 1 <= min(low_limit, len - 1) && (a.window <= 0 || high_limit - key0 < a.window);
                const float* const block_powers = powers + (j & 3) * 2 * Z::kKeys;
#pragma unroll 1
                for (int c = 0; c < Z::kKeys / 32; ++c) {
                    const auto load_scores = [&](uint32_t (&s)[32]) {
                        tmem_load32(s_at + 32 * c, s);
                        if constexpr (kOwn) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) s[i] = __float_as_uint(__uint_as_float(s[i]) * block_powers[32 * c + i]);
                        }
                        if (!whole) {
                            const int last = limit - key0 - 32 * c, first = from - key0 - 32 * c;
                            uint32_t hidden = 0;  // keys of blocks that are not there
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                if (missing >> (8 * (2 * c + i)) & 1) hidden |= 0xffffu << (16 * i);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (i > last || i < first || (hidden >> i & 1)) s[i] = 0xff800000u;  // -infinity
                        }
                    };
                    // rows that have outgrown their reference get another; what they have so far falls with it
                    const auto move_reference = [&](float now) {
                        const float fall = exp2_approx(ref - now);
                        ref = now, sum *= fall;
                        if (j > 0) {
                            bar_wait(o_done + 8 * mat, (j - 1) & 1, &dead);
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
                        }
                        tmem_stored();
#pragma unroll 1
                        for (int i = 0; i < c; ++i) {
                            uint32_t x[16];
                            tmem_load16(s_at + 16 * i, x);
#pragma unroll
                            for (int k = 0; k < 16; ++k) x[k] = as_word(__hmul2(as_half2(x[k]), __float2half2_rn(fall)));
                            tmem_store16(s_at + 16 * i, x);
                        }
                        tmem_stored();
                    };
                    uint32_t p[16];
                    float part;
                    if constexpr (!kOwn) {
                        uint32_t s[32];
                        load_scores(s);
#pragma unroll 1
                        for (int round = 0;; ++round) {
                            float even = 0.f, odds = 0.f;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float x = exp2_approx(fmaf(__uint_as_float(s[2 * i]), back, -ref)), y = exp2_approx(fmaf(__uint_as_float(s[2 * i + 1]), back, -ref));
                                even += x, odds += y;
                                p[i] = pack2(x, y, false);
                            }
                            part = even + odds;
                            if (round || !__any_sync(0xffffffffu, part > kBound)) break;
                            float top = -INFINITY;
#pragma unroll
                            for (int i = 0; i < 32; ++i) top = fmaxf(top, __uint_as_float(s[i]));
                            move_reference(part > kBound ? top * back - kStart : ref);
                        }
                    } else {
                        const float* const f = block_powers + Z::kKeys + 32 * c;
                        float weight = 0.f;  // the sum with V's powers
#pragma unroll 1
                        for (int round = 0;; ++round) {
                            uint32_t s[32];  // read again in the second round: kept, it would cost the registers that P takes
                            load_scores(s);
                            if (round) {
                                float top = -INFINITY;
#pragma unroll
                                for (int i = 0; i < 32; ++i) top = fmaxf(top, fmaf(__uint_as_float(s[i]), back, (float)((int)(__float_as_uint(f[i]) >> 23) - 127)));
                                move_reference(weight > kBound ? top - kStart : ref);
                            }
                            part = weight = 0.f;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float x = exp2_approx(fmaf(__uint_as_float(s[2 * i]), back, -ref)), y = exp2_approx(fmaf(__uint_as_float(s[2 * i + 1]), back, -ref));
                                const float u = x * f[2 * i], v = y * f[2 * i + 1];
                                part += x + y, weight += u + v;
                                p[i] = pack2(u, v, false);
                            }
                            if (round || !__any_sync(0xffffffffu, weight > kBound)) break;
                        }
                    }
                    sum += part;
                    tmem_store16(s_at + 16 * c, p);
                }
                tmem_stored();
                tmem_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full + 8 * mat);
            }
        };
        if (odd) make_p(std::true_type());
        else make_p(std::false_type());
        const bool some = blocks > 0 && mat < mats;
        if (some) {
            bar_wait(o_done + 8 * mat, (blocks - 1) & 1, &dead);
            __syncwarp();
            tmem_after();
        }
        // Whoever gave up said so before its next arrival, and outputs are behind all arrivals: none that went wrong gets here
        // without the mark.
        if (*static_cast<volatile int*>(&dead)) sum = __uint_as_float(0x7fc00000u);
        uint16_t* dst = a.out.data + (int64_t)(qs + token) * a.out.s_token + (int64_t)q_head * a.out.s_head;
        if (splits == 1) {
            const float inv = sum == 0.f ? 0.f : two_to(-kUpV) / sum;
#pragma unroll 1
            for (int i = 0; i < D; i += 32) {
                uint32_t o[32];
                if (some) {
                    tmem_load32(o_at + i, o);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0;
                }
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
            const bool rows_here = (tid & ~31) < rows;  // of this warp
#pragma unroll 1
            for (int i = 0; i < (rows_here ? D : 0); i += 32) {
                uint32_t o[32];
                if (some) {
                    tmem_load32(o_at + i, o);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0;
                }
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
                // 32 rows and 16 dims to a warp at a time, four parts' loads in flight
                const float* part = slots + (int64_t)(part_of - split) * Z::kPartFloats;
#pragma unroll 1
                for (int task = wid; task < (rows + 31) / 32 * (D / 16); task += kSoftmaxWarps) {
                    const int r = task / (D / 16) * 32 + lane, d = task % (D / 16) * 16;
                    const int my_row = row0 + min(r, rows - 1), my_token = prompt_token(a, my_row), my_head = head * a.group + my_row - my_token * a.group;
                    float f[kMostSplits], top = kUnset, all = 0.f;
#pragma unroll
                    for (int i = 0; i < kMostSplits; ++i) f[i] = i < splits ? __ldcg(part + (int64_t)i * Z::kPartFloats + D * kRows + r) : kUnset;
#pragma unroll
                    for (int i = 0; i < kMostSplits; ++i) top = fmaxf(top, f[i]);
#pragma unroll
                    for (int i = 0; i < kMostSplits; ++i) {
                        f[i] = exp2_approx(f[i] - top);
                        if (i < splits) all = fmaf(f[i], __ldcg(part + (int64_t)i * Z::kPartFloats + (D + 1) * kRows + r), all);
                    }
                    float o[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] = 0.f;
#pragma unroll
                    for (int i = 0; i < kMostSplits; ++i) {
                        if (i >= splits) break;
                        const float* x = part + (int64_t)i * Z::kPartFloats + d * kRows + r;
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = fmaf(f[i], __ldcg(x + k * kRows), o[k]);
                    }
                    const float inv = all == 0.f ? 0.f : two_to(-kUpV) / all;
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
    } else if (wid < kSoftmaxWarps + kUnpackWarps) {
        // ---- keys and values: a tile of every block to a warp ----
        const int w = wid - kSoftmaxWarps, g = lane >> 2, t = lane & 3;
        const int32_t* row = v.tables + (int64_t)seq * v.max_blocks;
        const uint8_t* slice = v.base + (int64_t)head * v.s_head;
        const int k_at0 = (w * kKvqTile + g) * 128 + (g << 4) + t * 4, v_at0 = (w / 4 * D + g) * 128 + ((w % 4 * 2 ^ g) << 4) + t * 4;
        RawK<D> rk;
        RawV<D> rv;
        const auto find = [&](int j) -> const uint8_t* {  // the warp's tile of block j
            const int key = first_key + j * Z::kKeys + w * kKvqTile, tile = key / kKvqTile;
            if (j >= blocks || key >= end) return nullptr;
            const int in_row = tile / v.block_tiles, id = __ldcg(row + in_row);
            if ((uint32_t)id < (uint32_t)v.nb) return slice + (int64_t)id * v.s_block + (tile - in_row * v.block_tiles) * (kKvqTile * kvq_token_bytes(D));
            if (lane == 0) kvq_error(v, kErrBadBlock);
            return nullptr;
        };
        const auto valid = [&](int j) { return len - (first_key + j * Z::kKeys + w * kKvqTile); };
        const uint8_t* at = find(0);
        load_k<D>(at, g, t, rk);
        load_v<D>(at ? at + v.s_kv : nullptr, valid(0), g, t, rv);
        look(w);
        const bool odd = all_meet();
        const auto unpack = [&](auto own) {
            constexpr bool kOwn = decltype(own)::value;
#pragma unroll 1
            for (int j = 0; j < blocks; ++j) {
                const int place_of = j & 1, turn = (j >> 1) & 1;
                const uint8_t* next = find(j + 1);
                if (j > 1) bar_wait(k_free + 8 * place_of, turn ^ 1, &dead);
                float down_k[2] = {two_to(kUpK), two_to(kUpK)}, down_v[4] = {two_to(kUpV), two_to(kUpV), two_to(kUpV), two_to(kUpV)};
                if constexpr (kOwn) {  // told to the warps that make P before K is
                    float* const my_powers = powers + (j & 3) * 2 * Z::kKeys + w * kKvqTile;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float f = at ? power_of<kUpK>(rk.par[h]) : 1.f;
                        down_k[h] = down_of<kUpK>(f);
                        if (t == 0) my_powers[g + 8 * h] = f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float f = power_of<kUpV>(rv.par[i]);
                        down_v[i] = down_of<kUpV>(f);
                        if (g == 0) my_powers[Z::kKeys + 2 * t + (i & 1) + (i >> 1) * 8] = f;
                    }
                }
                {
                    uint8_t* place[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) place[c] = sk + place_of * Z::kK + (k_at0 ^ (c << 4));
                    store_k<D>(place, rk, down_k);
                }
                for_tensor_cores();
                if (lane == 0) gone[j & 3][w] = at == nullptr;
                __syncwarp();
                if (lane == 0) bar_arrive(k_full + 8 * place_of);
                load_k<D>(next, g, t, rk);
                if (j > 1) bar_wait(v_free + 8 * place_of, turn ^ 1, &dead);
                {
                    uint8_t* const place[2] = {sv + place_of * Z::kV + v_at0, sv + place_of * Z::kV + (v_at0 ^ 16)};
                    store_v<D>(place, rv, down_v);
                }
                for_tensor_cores();
                __syncwarp();
                if (lane == 0) bar_arrive(v_full + 8 * place_of);
                load_v<D>(next ? next + v.s_kv : nullptr, valid(j + 1), g, t, rv);
                at = next;
            }
        };
        if (odd) unpack(std::true_type());
        else unpack(std::false_type());
    } else {
        // ---- matrix instructions: one lane issues them, three wait for what they need at the same time ----
        look(kUnpackWarps);
        all_meet();
        const uint32_t leads = lane == 0;
        const int n = __shfl_sync(0xffffffffu, blocks, 0), live = __shfl_sync(0xffffffffu, mats, 0);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint32_t q_low = operand_low((uint32_t)__cvta_generic_to_shared(sq)), k_low = operand_low((uint32_t)__cvta_generic_to_shared(sk)),
                       v_low = operand_low((uint32_t)__cvta_generic_to_shared(sv));
        if (blocks > 0) bar_wait(q_full, 0, &dead, a.tries);
        __syncwarp();
#pragma unroll 1
        for (int j = -1; j < n; ++j) {
            // P.V of block j and the scores of block j + 1, matrix by matrix: while one's run, P of the other is made. They run in
            // the order of issue, so the scores may take the place of the probabilities before them.
            const uint32_t place = j & 1, next = place ^ 1;
            const uint32_t v_block = v_low + place * (Z::kV >> 4), k_block = k_low + next * (Z::kK >> 4);
            const bool values = j >= 0, scores = j + 1 < n;
            if (lane == 1 ? scores : values)
                bar_wait(lane == 1 ? k_full + 8 * next : lane == 2 ? v_full + 8 * place : p_full, (lane == 1 ? j + 1 >> 1 : lane == 2 ? j >> 1 : j) & 1, &dead);
            __syncwarp();
#pragma unroll
            for (int mat = 0; mat < Z::kMats; ++mat) {
                if (mat >= live) break;
                const uint32_t s = tm + mat * Z::kKeys;
                if (values) {
                    if (mat > 0) {
                        bar_wait(p_full + 8 * mat, j & 1, &dead);
                        __syncwarp();
                    }
                    tmem_after();
#pragma unroll
                    for (int k = 0; k < Z::kKeys / 16; ++k)
                        mma_tmem<D>(tm + Z::kO + mat * D, s + 8 * k, v_block + ((k / 4) * (D * 128) + (k % 4) * 32 >> 4), k ? 1 : j, leads);
                    commit_to(o_done + 8 * mat, leads);
                }
                if (scores) {
                    if (!values) tmem_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_smem<Z::kKeys>(s, q_low + (mat * Z::kQ + (k / 4) * (kRowsM * 128) + (k % 4) * 32 >> 4),
                                           k_block + ((k / 4) * (Z::kKeys * 128) + (k % 4) * 32 >> 4), k > 0, leads);
                    commit_to(s_full + 8 * mat, leads);
                }
            }
            if (values) commit_to(v_free + 8 * place, leads);
            if (scores) commit_to(k_free + 8 * next, leads);
        }
        // Nothing stays in flight, whatever happened: a barrier of its own stands behind everything, since a block that gave up may
        // have run ahead of the others by several phases. Then the last arrival on each of these; block b is in place b & 1.
        __syncwarp();
        commit_to(all_done, leads);
        bar_drain(all_done, 1, &dead);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i < live) bar_drain(s_full + 8 * i, n, &dead), bar_drain(o_done + 8 * i, n, &dead);
            bar_drain(k_free + 8 * i, (n + 1 - i) >> 1, &dead), bar_drain(v_free + 8 * i, (n + 1 - i) >> 1, &dead);
        }
        __syncwarp();
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    __syncwarp();
    if (wid == kSoftmaxWarps + kUnpackWarps)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Z::kColumns));
    if (tid == 0 && dead) kvq_error(v, kErrWaitLimit);
}

template <int D>
cudaError_t launch(PromptArgs& a, bool bf, int sms, int max_rows, cudaStream_t stream) {
    using Z = Prompt<D>;
    a.row_blocks = (max_rows + Z::kRows - 1) / Z::kRows;
    const int64_t units = (int64_t)a.row_blocks * a.v.num_seqs * a.v.kv_heads;
    // a unit is a thread block's work; those that are left when the others have filled the GPU whole times share it, each
    // one's keys split (2048 queries over 8191 keys on 148 SMs: 512 units, 68 of them in two parts each)
    constexpr int kParts = (int)((kAttendWorkspace - kAttendCounterBytes) / (Z::kPartFloats * 4));
    const int places = std::min(sms, kParts);
    const int64_t rest = units % sms;
    a.splits = rest ? (int)std::min<int64_t>(kMostSplits, places / rest) : 1;
    if (a.splits < 2) a.splits = 1;
    a.whole = (int)(a.splits > 1 ? units - rest : units);
    static_assert(kParts >= 148 && kParts <= 2 * kAttendMaxCtas, "workspace");  // splits of two at least: a counter for two parts
    if (units > 0x7fffffff / kMostSplits) return cudaErrorInvalidConfiguration;
    a.tries = prompt_wait_tries();
    return launch_after(bf ? kvq_prompt_kernel<D, true> : kvq_prompt_kernel<D, false>, a.whole + (units - a.whole) * a.splits, Z::kThreads, Z::kBytes, stream, a);
}

}  // namespace

int32_t prompt_wait_tries() { return g_wait_tries.load(std::memory_order_relaxed); }

cudaError_t launch_prompt(const KvqView& v, const KvqRows& q, const KvqRows& out, float* lse, void* workspace, float scale_log2, int32_t head_dim,
                          int32_t q_heads, int32_t group, uint32_t by_group, int32_t window, int32_t room, bool bf, int sms, int32_t max_rows,
                          cudaStream_t stream) {
    PromptArgs a{v, q, out, lse, static_cast<uint8_t*>(workspace), scale_log2, group, q_heads, window, room, by_group, 0, 0, 1, kWaitTries};
    return head_dim == 64 ? launch<64>(a, bf, sms, max_rows, stream)
           : head_dim == 128 ? launch<128>(a, bf, sms, max_rows, stream) : launch<256>(a, bf, sms, max_rows, stream);
}

}  // namespace remp

extern "C" void remp_kvq_set_wait_limit(int32_t tries) {
    remp::g_wait_tries.store(tries < 0 ? remp::kWaitTries : std::min(tries, remp::kWaitTries), std::memory_order_relaxed);
}
