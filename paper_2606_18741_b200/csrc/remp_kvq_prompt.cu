// Attention over the 4-bit cache for many queries per sequence (prompts and their chunks), on the tensor cores' own memory.
//
// Mathematics: softmax(scale * q.K^T + mask).V, one thread block for 128 rows (tokens x query heads of one KV head) and a
// range of the keys, block by block of kKeys keys: S = Q.K^T, P = 2^(S*back - ref), O += P.V, with a running reference for
// each row that moves only when the probabilities of 32 keys outgrow kBound.
// Rounding: q is exact in half after a power of two per row; keys and values s*c + m are rounded to half (a quarter of them,
// so that every 16-bit input stays finite) and so is P; S, O, sums and references are in 32 bits.
//
// Bound: tensor cores (4*D flops for each row and key), then issue slots: four warps turn codes into halves, four compute
// P, one thread issues the matrix instructions; two thread blocks to an SM take turns on the tensor cores. Q, K and V^T lie in
// shared memory in rows of 128 bytes, 16-byte pieces exchanged within 8 rows (piece ^ (row & 7)); K's codes are stored so
// that a word gives neighbouring dims and V's words of two tokens give a pair of keys, so each 4-byte store of a warp meets
// 32 different banks. S and P share their columns of the tensor memory, O has its own.
//
// Order: K of the next block is made while P of this one is computed (its place is free once S is complete), V while the
// next S is. Every wait is on a barrier in shared memory and bounded: a block that gives up sets error bit 4, goes on
// without waiting, and ends.

#include "remp_kvq_device.h"

namespace remp {

namespace {

constexpr int kRowsM = 128;
constexpr int kSoftmaxWarps = 4, kUnpackWarps = 4, kPromptThreads = (kSoftmaxWarps + kUnpackWarps + 1) * 32;
constexpr float kUnset = -1e30f;     // reference of a row that has seen nothing
constexpr float kBound = 16384.f;    // of the sum of 32 probabilities
constexpr float kStart = 8.f;        // log2 of the largest probability when a reference is set
constexpr uint32_t kWaitTries = 1u << 18;

template <int D>
struct Prompt {
    static constexpr int kKeys = D == 256 ? 64 : 128, kTiles = kKeys / kKvqTile, kWarpTiles = kTiles / kUnpackWarps;
    static constexpr int kQ = kRowsM * D * 2, kK = kKeys * D * 2, kV = kKeys * D * 2;  // bytes
    static constexpr int kBytes = kQ + kK + kV + 1024;
    static constexpr int kColumns = D == 256 ? 512 : 256, kO = kKeys;  // of the tensor memory: S and P from 0, O behind
    static constexpr int kCtas = D == 256 ? 1 : 2;
    static constexpr int kPartFloats = kRowsM * (D + 2);
};

// ---- barriers and tensor memory ----

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
// Bounded: a wait that runs out marks the block, and nothing in it waits any more.
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
    for (uint32_t i = 0; i < kWaitTries; ++i) {
        if (bar_try(bar, parity)) return;
        if (*dead) return;
    }
    *dead = 1;
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit_to(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Rows of 128 bytes, 16-byte pieces exchanged within 8 rows: a matrix of 64 halves a row, rows along M or N.
__device__ __forceinline__ uint64_t operand(uint32_t at) {
    return (uint64_t)(at >> 4 & 0x3fff) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// halves times halves into 32 bits, 128 rows, n columns, both operands along K
__host__ __device__ constexpr uint32_t shape_of(int n) { return 1u << 4 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRowsM >> 4) << 24; }

__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b),
                 "r"(shape), "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b),
                 "r"(shape), "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void for_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

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
    int32_t row_blocks, splits;  // of a sequence and KV head at most; parts of its keys
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

// Rows of K, a key each: place[c] is where piece c of this lane's 8 keys' rows begins, for its words of the pieces. i: the
// tile of the warp's.
template <int D>
__device__ __forceinline__ void store_k(uint8_t* const (&place)[8], int i, const RawK<D>& r) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int grp = 0; grp < D / 64; ++grp) {
            const float s = bf_low(r.par[h][grp]) * 0.25f, m = bf_high(r.par[h][grp]) * 0.25f;
            const __half2 step = finite_halves(s, s), low = finite_halves(m, m);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint32_t z[4];
                four_halves(r.w[h][2 * grp + x], step, low, z);
#pragma unroll
                for (int b = 0; b < 4; ++b) *reinterpret_cast<uint32_t*>(place[4 * x + b] + (i * kKvqTile + 8 * h + grp * Prompt<D>::kKeys) * 128) = z[b];
            }
        }
}

// Rows of V^T, a dim each: row 8n + g from `place` on, two keys to a word.
template <int D>
__device__ __forceinline__ void store_v(uint8_t* const (&place)[2], const RawV<D>& r) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int grp = 0; grp < D / 64; ++grp) {
            const uint32_t p0 = r.par[2 * h][grp], p1 = r.par[2 * h + 1][grp];
            const __half2 step = finite_halves(bf_low(p0) * 0.25f, bf_low(p1) * 0.25f), low = finite_halves(bf_high(p0) * 0.25f, bf_high(p1) * 0.25f);
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
__global__ void __launch_bounds__(kPromptThreads, Prompt<D>::kCtas) kvq_prompt_kernel(const __grid_constant__ PromptArgs a) {
    using Z = Prompt<D>;
    extern __shared__ uint8_t smem_[];
    __shared__ __align__(8) uint64_t bars[6];
    __shared__ uint32_t tmem_at;
    __shared__ int dead;
    __shared__ int is_last;
    __shared__ __align__(4) uint8_t gone[2][kUnpackWarps];  // of a block of keys: bit i, tile i of the warp's is not there

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const KvqView& v = a.v;
    grid_begin();

    // ---- this block's rows and keys ----
    // row blocks from the last to the first: the last sees the most keys
    int unit = blockIdx.x;
    const int split = unit % a.splits;
    unit /= a.splits;
    const int head = unit % v.kv_heads;
    unit /= v.kv_heads;
    const int seq = unit % v.num_seqs, block = a.row_blocks - 1 - unit / v.num_seqs;
    const int qs = max(0, v.query_start[seq]), qe = min(v.num_tokens, v.query_start[seq + 1]);
    const int queries = max(0, qe - qs), rows_all = queries * a.group, row0 = block * kRowsM;
    if (row0 >= rows_all) return;
    const int rows = min(kRowsM, rows_all - row0), len_ = v.seq_lens[seq], len = min(max(len_, 0), a.room);
    if (len != len_ && tid == 0) kvq_error(v, kErrBadLength);
    const int first_pos = len_ - queries;
    const int low_limit = first_pos + prompt_token(a, row0), high_limit = first_pos + prompt_token(a, row0 + rows - 1);
    const int end = max(0, min(len, high_limit + 1)), begin = min(end, a.window > 0 ? max(0, low_limit - a.window + 1) : 0) / kKvqTile * kKvqTile;
    const int blocks_all = (end - begin + Z::kKeys - 1) / Z::kKeys;
    const int b0 = (int)((long long)blocks_all * split / a.splits), b1 = (int)((long long)blocks_all * (split + 1) / a.splits);
    const int blocks = b1 - b0, first_key = begin + b0 * Z::kKeys;

    uint8_t* smem = smem_ + ((1024u - ((uint32_t)__cvta_generic_to_shared(smem_) & 1023u)) & 1023u);
    uint8_t *sq = smem, *sk = smem + Z::kQ, *sv = sk + Z::kK;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars);
    const uint32_t k_full = bar, v_full = bar + 8, s_full = bar + 16, p_full = bar + 24, o_done = bar + 32, q_full = bar + 40;
    if (tid == 0) {
        bar_init(k_full, kUnpackWarps), bar_init(v_full, kUnpackWarps), bar_init(s_full, 1), bar_init(p_full, kSoftmaxWarps), bar_init(o_done, 1);
        bar_init(q_full, kSoftmaxWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead = 0, is_last = 0;
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

    if (wid < kSoftmaxWarps) {
        // ---- P and the output: one row to a thread ----
        const uint32_t lanes = tmem + ((uint32_t)(wid * 32) << 16);
        const int row = row0 + min(tid, rows - 1), token = prompt_token(a, row), q_head = head * a.group + row - token * a.group;
        const bool real = tid < rows;
        const int limit = min(first_pos + token, len - 1), from = a.window > 0 ? first_pos + token - a.window + 1 : 0;
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
            const int e = most ? max(-120, min(93, 3 - ((int)(__float_as_uint(top) >> 23) - 127))) : 0;
            const float up = __uint_as_float((uint32_t)(127 + e) << 23);
            back = a.scale_log2 * 4.f * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll 4
            for (int i = 0; i < D / 8; ++i) {
                const uint4 x = reinterpret_cast<const uint4*>(src)[i];
                uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 f = BF ? make_float2(bf_low(w[k]), bf_high(w[k])) : __half22float2(as_half2(w[k]));
                    w[k] = pack2(f.x * up, f.y * up, false);
                }
                *reinterpret_cast<uint4*>(sq + (i / 8) * (kRowsM * 128) + tid * 128 + (((i % 8) ^ (tid & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            for_tensor_cores();
            __syncwarp();
            if (lane == 0) bar_arrive(q_full);
        }
        float ref = kUnset, sum = 0.f;
#pragma unroll 1
        for (int j = 0; j < blocks; ++j) {
            bar_wait(s_full, j & 1, &dead);
            tmem_after();
            const int key0 = first_key + j * Z::kKeys;
            const uint32_t missing = *reinterpret_cast<const volatile uint32_t*>(gone[j & 1]);
            const bool whole = missing == 0 && key0 + Z::kKeys - 1 <= min(low_limit, len - 1) && (a.window <= 0 || key0 > high_limit - a.window);
#pragma unroll 1
            for (int c = 0; c < Z::kKeys / 32; ++c) {
                uint32_t s[32];
                tmem_load32(lanes + 32 * c, s);
                if (!whole) {
                    const int last = limit - key0 - 32 * c, first = from - key0 - 32 * c;
                    uint32_t hidden = 0;  // keys of blocks that are not there
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int tile = 2 * c + i;
                        if (missing >> (tile / Z::kWarpTiles * 8 + tile % Z::kWarpTiles) & 1) hidden |= 0xffffu << (16 * i);
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (i > last || i < first || (hidden >> i & 1)) s[i] = 0xff800000u;  // -infinity
                }
                uint32_t p[16];
                float part;
#pragma unroll 1
                for (int round = 0;; ++round) {
                    float even = 0.f, odd = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float x = exp2_approx(fmaf(__uint_as_float(s[2 * i]), back, -ref)), y = exp2_approx(fmaf(__uint_as_float(s[2 * i + 1]), back, -ref));
                        even += x, odd += y;
                        p[i] = pack2(x, y, false);
                    }
                    part = even + odd;
                    if (round || !__any_sync(0xffffffffu, part > kBound)) break;
                    // rows that have outgrown their reference get another; what they have so far falls with it
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 32; ++i) top = fmaxf(top, __uint_as_float(s[i]));
                    const float now = part > kBound ? top * back - kStart : ref, fall = exp2_approx(ref - now);
                    ref = now, sum *= fall;
                    if (j > 0) {
                        bar_wait(o_done, (j - 1) & 1, &dead);
                        tmem_after();
#pragma unroll 1
                        for (int i = 0; i < D; i += 16) {
                            uint32_t o[16];
                            tmem_load16(lanes + Z::kO + i, o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * fall);
                            tmem_store16(lanes + Z::kO + i, o);
                        }
                    }
                    tmem_stored();
#pragma unroll 1
                    for (int i = 0; i < c; ++i) {
                        uint32_t x[16];
                        tmem_load16(lanes + 16 * i, x);
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = as_word(__hmul2(as_half2(x[k]), __float2half2_rn(fall)));
                        tmem_store16(lanes + 16 * i, x);
                    }
                    tmem_stored();
                }
                sum += part;
                tmem_store16(lanes + 16 * c, p);
            }
            tmem_stored();
            tmem_before();
            __syncwarp();
            if (lane == 0) bar_arrive(p_full);
        }
        if (blocks > 0) {
            bar_wait(o_done, (blocks - 1) & 1, &dead);
            tmem_after();
        }
        uint16_t* dst = a.out.data + (int64_t)(qs + token) * a.out.s_token + (int64_t)q_head * a.out.s_head;
        if (a.splits == 1) {
            const float inv = sum == 0.f ? 0.f : 4.f / sum;
#pragma unroll 1
            for (int i = 0; i < D; i += 32) {
                uint32_t o[32];
                if (blocks > 0) {
                    tmem_load32(lanes + Z::kO + i, o);
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
            float* mine = slots + (int64_t)blockIdx.x * Z::kPartFloats;
#pragma unroll 1
            for (int i = 0; i < D; i += 32) {
                uint32_t o[32];
                if (blocks > 0) {
                    tmem_load32(lanes + Z::kO + i, o);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0;
                }
#pragma unroll
                for (int k = 0; k < 32; ++k) mine[(i + k) * kRowsM + tid] = __uint_as_float(o[k]);
            }
            mine[D * kRowsM + tid] = ref, mine[(D + 1) * kRowsM + tid] = sum;
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (tid == 0) {
                uint32_t* counter = reinterpret_cast<uint32_t*>(a.workspace) + blockIdx.x / a.splits;
                uint32_t before;
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
                is_last = before == (uint32_t)a.splits - 1;
                if (is_last) *counter = 0;  // ready for the next call
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (is_last) {
                const float* part = slots + (int64_t)(blockIdx.x - split) * Z::kPartFloats;
                float top = kUnset;
#pragma unroll 4
                for (int i = 0; i < a.splits; ++i) top = fmaxf(top, __ldcg(part + (int64_t)i * Z::kPartFloats + D * kRowsM + tid));
                float all = 0.f;
#pragma unroll 4
                for (int i = 0; i < a.splits; ++i)
                    all = fmaf(exp2_approx(__ldcg(part + (int64_t)i * Z::kPartFloats + D * kRowsM + tid) - top),
                               __ldcg(part + (int64_t)i * Z::kPartFloats + (D + 1) * kRowsM + tid), all);
                const float inv = all == 0.f ? 0.f : 4.f / all;
#pragma unroll 1
                for (int d = 0; d < D; d += 8) {
                    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
                    for (int i = 0; i < a.splits; ++i) {
                        const float* x = part + (int64_t)i * Z::kPartFloats;
                        const float f = exp2_approx(__ldcg(x + D * kRowsM + tid) - top);
#pragma unroll
                        for (int k = 0; k < 8; ++k) o[k] = fmaf(f, __ldcg(x + (d + k) * kRowsM + tid), o[k]);
                    }
                    uint32_t w[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) w[x] = pack2(o[2 * x] * inv, o[2 * x + 1] * inv, BF);
                    if (real) *reinterpret_cast<uint4*>(dst + d) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                if (real && a.lse) a.lse[(int64_t)(qs + token) * a.q_heads + q_head] = all == 0.f ? -INFINITY : (top + log2f(all)) * 0.69314718055994531f;
            }
        }
    } else if (wid < kSoftmaxWarps + kUnpackWarps) {
        // ---- keys and values: kWarpTiles tiles of a block to a warp ----
        const int w = wid - kSoftmaxWarps, g = lane >> 2, t = lane & 3;
        const int32_t* row = v.tables + (int64_t)seq * v.max_blocks;
        const uint8_t* slice = v.base + (int64_t)head * v.s_head;
        RawK<D> rk[Z::kWarpTiles];
        RawV<D> rv[Z::kWarpTiles];
        const uint8_t* at[Z::kWarpTiles];
        const auto find = [&](int j) {  // where the tiles of block j are
#pragma unroll
            for (int i = 0; i < Z::kWarpTiles; ++i) {
                const int key = first_key + j * Z::kKeys + (w * Z::kWarpTiles + i) * kKvqTile, tile = key / kKvqTile;
                at[i] = nullptr;
                if (j < blocks && key < end) {
                    const int in_row = tile / v.block_tiles, id = __ldcg(row + in_row);
                    if ((uint32_t)id < (uint32_t)v.nb) at[i] = slice + (int64_t)id * v.s_block + (tile - in_row * v.block_tiles) * (kKvqTile * kvq_token_bytes(D));
                    else if (lane == 0) kvq_error(v, kErrBadBlock);
                }
            }
        };
        const auto absent = [&]() {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < Z::kWarpTiles; ++i) m |= at[i] ? 0u : 1u << i;
            return (uint8_t)m;
        };
        const auto valid = [&](int j, int i) { return len - (first_key + j * Z::kKeys + (w * Z::kWarpTiles + i) * kKvqTile); };
        find(0);
        uint8_t away = absent();
#pragma unroll
        for (int i = 0; i < Z::kWarpTiles; ++i) load_k<D>(at[i], g, t, rk[i]);
#pragma unroll
        for (int i = 0; i < Z::kWarpTiles; ++i) load_v<D>(at[i] ? at[i] + v.s_kv : nullptr, valid(0, i), g, t, rv[i]);
#pragma unroll 1
        for (int j = 0; j < blocks; ++j) {
            find(j + 1);
            if (j > 0) bar_wait(s_full, (j - 1) & 1, &dead);
            {
                uint8_t* place[8];
                const int at0 = (w * Z::kWarpTiles * kKvqTile + g) * 128 + (g << 4) + t * 4;
#pragma unroll
                for (int c = 0; c < 8; ++c) place[c] = sk + (at0 ^ (c << 4));
#pragma unroll
                for (int i = 0; i < Z::kWarpTiles; ++i) store_k<D>(place, i, rk[i]);
            }
            for_tensor_cores();
            if (lane == 0) gone[j & 1][w] = away;
            __syncwarp();
            if (lane == 0) bar_arrive(k_full);
            away = absent();
#pragma unroll
            for (int i = 0; i < Z::kWarpTiles; ++i) load_k<D>(at[i], g, t, rk[i]);
            if (j > 0) bar_wait(o_done, (j - 1) & 1, &dead);
#pragma unroll
            for (int i = 0; i < Z::kWarpTiles; ++i) {
                const int tile = w * Z::kWarpTiles + i, at0 = (tile / 4 * D + g) * 128 + ((tile % 4 * 2 ^ g) << 4) + t * 4;
                uint8_t* const place[2] = {sv + at0, sv + (at0 ^ 16)};
                store_v<D>(place, rv[i]);
            }
            for_tensor_cores();
            __syncwarp();
            if (lane == 0) bar_arrive(v_full);
#pragma unroll
            for (int i = 0; i < Z::kWarpTiles; ++i) load_v<D>(at[i] ? at[i] + v.s_kv : nullptr, valid(j + 1, i), g, t, rv[i]);
        }
    } else if (lane == 0 && blocks > 0) {
        // ---- matrix instructions ----
        const uint32_t q_at = (uint32_t)__cvta_generic_to_shared(sq), k_at = (uint32_t)__cvta_generic_to_shared(sk), v_at = (uint32_t)__cvta_generic_to_shared(sv);
        const auto scores = [&](int j) {
            bar_wait(k_full, j & 1, &dead);
            tmem_after();
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                mma_smem(tmem, operand(q_at + (k / 4) * (kRowsM * 128) + (k % 4) * 32), operand(k_at + (k / 4) * (Z::kKeys * 128) + (k % 4) * 32),
                         shape_of(Z::kKeys), k > 0);
            commit_to(s_full);
        };
        bar_wait(q_full, 0, &dead);
        scores(0);
#pragma unroll 1
        for (int j = 0; j < blocks; ++j) {
            bar_wait(v_full, j & 1, &dead);
            bar_wait(p_full, j & 1, &dead);
            tmem_after();
#pragma unroll
            for (int k = 0; k < Z::kKeys / 16; ++k)
                mma_tmem(tmem + Z::kO, tmem + 8 * k, operand(v_at + (k / 4) * (D * 128) + (k % 4) * 32), shape_of(D), j > 0 || k > 0);
            commit_to(o_done);
            if (j + 1 < blocks) {
                bar_wait(o_done, j & 1, &dead);  // the next scores take the place of these probabilities
                scores(j + 1);
            }
        }
        for (uint32_t i = 0; i < kWaitTries && !bar_try(o_done, (blocks - 1) & 1); ++i) {}  // nothing stays in flight, whatever happened
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
    a.row_blocks = (max_rows + kRowsM - 1) / kRowsM;
    const int64_t units = (int64_t)a.row_blocks * a.v.num_seqs * a.v.kv_heads;
    // too few units to fill the GPU: each one's keys are split, one part to a thread block
    constexpr int kParts = (int)((kAttendWorkspace - kAttendCounterBytes) / (Z::kPartFloats * 4));
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>(16, std::min(sms * Z::kCtas, kParts) / units));
    static_assert(kParts >= 148 * Z::kCtas && kParts <= 2 * kAttendMaxCtas, "workspace");  // splits of two at least: a counter for two parts
    if (units > 0x7fffffff / 16) return cudaErrorInvalidConfiguration;
    return launch_after(bf ? kvq_prompt_kernel<D, true> : kvq_prompt_kernel<D, false>, units * a.splits, kPromptThreads, Z::kBytes, stream, a);
}

}  // namespace

cudaError_t launch_prompt(const KvqView& v, const KvqRows& q, const KvqRows& out, float* lse, void* workspace, float scale_log2, int32_t head_dim,
                          int32_t q_heads, int32_t group, uint32_t by_group, int32_t window, int32_t room, bool bf, int sms, int32_t max_rows,
                          cudaStream_t stream) {
    PromptArgs a{v, q, out, lse, static_cast<uint8_t*>(workspace), scale_log2, group, q_heads, window, room, by_group, 0, 1};
    return head_dim == 64 ? launch<64>(a, bf, sms, max_rows, stream)
           : head_dim == 128 ? launch<128>(a, bf, sms, max_rows, stream) : launch<256>(a, bf, sms, max_rows, stream);
}

}  // namespace remp
