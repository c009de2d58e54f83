// Pieces of attention over a tile of 16 tokens of the 4-bit cache, one warp: fetch, queries, scores, values.
// Lane (g, t) = (lane / 4, lane % 4), as the matrix instructions number rows and columns.
#pragma once

#include <algorithm>

#include "remp_kvq.h"
#include "remp_launch.h"

namespace remp {

constexpr int kAttendMaxCtas = 512;
constexpr size_t kAttendCounterBytes = kAttendMaxCtas * 4;
constexpr size_t kAttendWorkspace = kAttendCounterBytes + (size_t)300 * 128 * (128 + 2) * 4;  // parts of prompts are the largest

// remp_kvq_prompt.cu: many queries of a sequence
cudaError_t launch_prompt(const KvqView& v, const KvqRows& q, const KvqRows& out, float* lse, void* workspace, float scale_log2, int32_t head_dim,
                          int32_t q_heads, int32_t group, uint32_t by_group, int32_t window, int32_t room, bool bf, int sms, int32_t max_rows,
                          cudaStream_t stream);

#ifdef __CUDACC__

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// d[16][8] += a[16][16] . b[16][8], halves into 32 bits
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// d = a . b
__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 8 x 8 halves, row g in lanes 4g..4g+3 (columns 2t, 2t+1 in lane t): rows become columns.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, bool bf) {
    if (bf) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A step is two tiles; in shared memory it is the codes of K (tile 0, tile 1), the codes of V, and the parameters of K and
// of V, so that every lane copies whole rounds of 16 bytes. The pieces of V's codes change places within 128 bytes
// (piece ^ (token & 6)): the lanes of a warp, which read four tokens' rows at once, then meet different banks.
template <int D>
struct KvqStep {
    static constexpr int kCodes = kKvqTile * D / 2, kParams = kKvqTile * D / 16;  // bytes of a tile of K or of V
    static constexpr int kK = 0, kV = 2 * kCodes, kParK = 4 * kCodes, kParV = kParK + 2 * kParams;
    static constexpr int kBytes = kParV + 2 * kParams;
};

// src0, src1: the tiles of K, their tiles of V `kv` bytes behind; there0, there1: whether they are.
template <int D>
__device__ __forceinline__ void kvq_fetch_step(const uint8_t* src0, const uint8_t* src1, bool there0, bool there1, int64_t kv, uint32_t dst, int lane) {
    using S = KvqStep<D>;
#pragma unroll
    for (int j = 0; j < 2; ++j)
        if (j ? there1 : there0) {
            const uint8_t* k = (j ? src1 : src0) + lane * 16;
            const uint8_t* v = k + kv;
#pragma unroll
            for (int i = 0; i < S::kCodes / 512; ++i) {
                const int swap = ((lane + 32 * i) / (D / 32)) & 6;
                cp_async16(dst + S::kK + j * S::kCodes + i * 512 + lane * 16, k + i * 512);
                cp_async16(dst + S::kV + j * S::kCodes + i * 512 + (lane ^ swap) * 16, v + i * 512);
            }
        }
#pragma unroll
    for (int i = 0; i < (D / 4 + 31) / 32; ++i) {
        const int p = lane + 32 * i, part = p / (D / 16);  // K of tile 0, of tile 1, V of tile 0, of tile 1
        const uint8_t* from = (part & 1 ? src1 : src0) + (part & 2 ? kv : 0) + S::kCodes + p % (D / 16) * 16;
        if ((D >= 128 || p < D / 4) && (part & 1 ? there1 : there0)) cp_async16(dst + S::kParK + p * 16, from);
    }
}

// This lane's 16-bit queries of one row (src points at dim 2t): words of dims 16i + 8h + 2t, +1.
template <int D>
__device__ __forceinline__ void kvq_load_queries(const uint16_t* src, bool real, uint32_t (&qf)[D / 16][2]) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) qf[i][h] = real ? *reinterpret_cast<const uint32_t*>(src + 16 * i + 8 * h) : 0u;
}

// Makes them the operand columns, in halves. Slots 0..7 of each 16 dims are taken 16-fold: they meet codes at bits 0..3, the
// others codes at bits 4..7. A power of two brings the row's largest value to [8, 16), so that halves hold 16-bit
// queries of any size from 2^-117 on exactly (down to 2^-28 of the largest). qsum: what codes of 1 in every dim would score in each
// group (the sums of the queries, in the units of a score); back: what a score is multiplied with; both for columns 2t and 2t+1.
// Rows of very large queries (2^115 at a scale of 128^-0.5) have a negative `back`: its 2^20 does not fit into it, and the
// scores have to take it before they meet -back.
template <int D>
__device__ __forceinline__ void kvq_make_queries(bool bf, int t, uint32_t (&qf)[D / 16][2], float (&qsum)[D / kKvqGroup][2],
                                                 float (&back)[2], float scale_log2) {
    uint32_t most = 0;  // both halves: the largest magnitude's bits
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) most = __vmaxu2(most, qf[i][h] & 0x7fff7fffu);
    most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 2));
    most = max(most >> 16, most & 0xffffu);
    const float top = bf ? __uint_as_float(most << 16) : __half2float(__ushort_as_half((unsigned short)most));
    // 2^e with top * 2^e in [8, 16); rows of 0 and rows beyond 2^123 or below 2^-117 keep a bounded exponent
    const int exponent = (int)(__float_as_uint(top) >> 23) - 127;
    const int e = most ? max(-120, min(120, 3 - exponent)) : 0;
    const float up = __uint_as_float((uint32_t)(127 + e) << 23), up16 = 16.f * up;
    const float plain = scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23), lifted = plain * 1048576.f;  // codes counted 2^-20
    const float down = lifted <= 3.402823466e38f ? fmaxf(lifted, 1.2e-38f) : -plain;
    float sums[D / kKvqGroup];
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w = qf[i][h];
            const float2 f = bf ? make_float2(bf_low(w), bf_high(w)) : __half22float2(*reinterpret_cast<const __half2*>(&w));
            sums[i / 4] = (i % 4 || h ? sums[i / 4] : 0.f) + (f.x + f.y);
            qf[i][h] = pack2(f.x * (h ? up : up16), f.y * (h ? up : up16), false);
        }
#pragma unroll
    for (int grp = 0; grp < D / kKvqGroup; ++grp) {  // in 32 bits: the matrix instructions' own sums are cut at every step
        sums[grp] += __shfl_xor_sync(0xffffffffu, sums[grp], 1);
        sums[grp] += __shfl_xor_sync(0xffffffffu, sums[grp], 2);
        sums[grp] *= up * 9.5367431640625e-7f;
#pragma unroll
        for (int c = 0; c < 2; ++c) qsum[grp][c] = __shfl_sync(0xffffffffu, sums[grp], (2 * t + c) * 4);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) back[c] = __shfl_sync(0xffffffffu, down, (2 * t + c) * 4);
}

// The steps and minima of tokens g (h = 0) and g+8 of a tile, one word for each group.
template <int D>
__device__ __forceinline__ void kvq_params(const uint8_t* params, int g, uint32_t (&par)[2][D / kKvqGroup]) {
    constexpr int G = D / kKvqGroup;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint8_t* p = params + (g + 8 * h) * (D / 16);
        if constexpr (G == 1) {
            par[h][0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (G == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            par[h][0] = x.x, par[h][1] = x.y;
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(p);
            par[h][0] = x.x, par[h][1] = x.y, par[h][2] = x.z, par[h][3] = x.w;
        }
    }
}

// s[n]: scores of tokens g (elements 0, 1) and g+8 (2, 3) with columns 8n + 2t, +1, before `back`.
template <int D, int NT>
__device__ __forceinline__ void kvq_scores(const uint8_t* codes, const uint8_t* params, int g, int t, const uint32_t (&qf)[NT][D / 16][2],
                                           const float (&qsum)[NT][D / kKvqGroup][2], float (&s)[NT][4]) {
    constexpr int G = D / kKvqGroup, W = D / 32;  // groups, words of a lane's row
    uint32_t w[2][W], par[2][G];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint8_t* row = codes + (g + 8 * h) * (D / 2) + t * (D / 8);
        if constexpr (W == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(row);
            w[h][0] = x.x, w[h][1] = x.y;
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const uint4 x = *reinterpret_cast<const uint4*>(row + 4 * i);
                w[h][i] = x.x, w[h][i + 1] = x.y, w[h][i + 2] = x.z, w[h][i + 3] = x.w;
            }
        }
    }
    kvq_params<D>(params, g, par);
#pragma unroll
    for (int grp = 0; grp < G; ++grp) {
        float acc[NT][4];
#pragma unroll
        for (int i = 2 * grp; i < 2 * grp + 2; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // dims 32i + 16h .. +15
                const uint32_t x0 = h ? w[0][i] >> 8 : w[0][i], x1 = h ? w[1][i] >> 8 : w[1][i];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t a0 = x0 & 0x000f000fu, a1 = x1 & 0x000f000fu, a2 = x0 & 0x00f000f0u, a3 = x1 & 0x00f000f0u;
                    if (i == 2 * grp && h == 0) mma16816_first(acc[n], a0, a1, a2, a3, qf[n][2 * i + h][0], qf[n][2 * i + h][1]);
                    else mma16816(acc[n], a0, a1, a2, a3, qf[n][2 * i + h][0], qf[n][2 * i + h][1]);
                }
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float step = bf_low(par[e >> 1][grp]), low = bf_high(par[e >> 1][grp]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float x = fmaf(low, qsum[n][grp][e & 1], grp ? s[n][e] : 0.f);
                s[n][e] = fmaf(step, acc[n][e], x);
            }
        }
    }
}

// c - 8 (codes at bits 0..3 of each half) or 16 (c - 8) (at bits 4..7), as halves: 1024 + c has the code in its last bits.
__device__ __forceinline__ uint32_t centred(uint32_t x, bool upper) {
    uint32_t y;  // one instruction takes the bits and sets the others
    if (upper) asm("lop3.b32 %0, %1, 0x00f000f0, %2, 0xea;" : "=r"(y) : "r"(x), "r"(0x64006400u));
    else asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(y) : "r"(x), "r"(0x64006400u));
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&y), __half2half2(__ushort_as_half(upper ? 0x6480 : 0x6408)));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// o += (V's codes - 8)^T . R^T (16-fold in rows g+8 of each 16 dims), where R = p * step rounded to half; low += sums of
// p * (minimum + 8 step); so sum p*v = o + low. Codes around 0 keep the sums of a long sequence small: the matrix
// instructions' sums are cut, not rounded, and over 100 thousand tokens codes of one sign put the result off by 2^-18
// of sum p*v's terms; what rounding R does is halved as well. p: the probabilities in kvq_scores' layout; par: kvq_params of the tile, 0
// for tokens that are not there.
template <int D, int NT>
__device__ __forceinline__ void kvq_values(const uint8_t* codes, int g, int t, const float (&p)[NT][4],
                                           const uint32_t (&par)[2][D / kKvqGroup], float (&o)[NT][D / 16][4],
                                           float (&low)[NT][D / kKvqGroup][2]) {
    constexpr int G = D / kKvqGroup;
    uint32_t w[4][G];  // tokens 2t, 2t+1, 2t+8, 2t+9: this lane's dims of each group
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = ((2 * t + (j & 1) + (j >> 1) * 8) * (D / 2) + g * (D / 16)) ^ ((2 * t) << 4);
        if constexpr (G == 1) {
            w[j][0] = *reinterpret_cast<const uint32_t*>(codes + at);
        } else if constexpr (G == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(codes + at);
            w[j][0] = x.x, w[j][1] = x.y;
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(codes + at);
            w[j][0] = x.x, w[j][1] = x.y, w[j][2] = x.z, w[j][3] = x.w;
        }
    }
#pragma unroll
    for (int grp = 0; grp < G; ++grp) {
        uint32_t b[NT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float step = bf_low(par[h][grp]), middle = fmaf(8.f, step, bf_high(par[h][grp]));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                b[n][h] = transpose8(pack2(p[n][2 * h] * step, p[n][2 * h + 1] * step, false));
                low[n][grp][0] = fmaf(p[n][2 * h], middle, low[n][grp][0]);
                low[n][grp][1] = fmaf(p[n][2 * h + 1], middle, low[n][grp][1]);
            }
        }
        const uint32_t x[2] = {__byte_perm(w[0][grp], w[1][grp], 0x5410), __byte_perm(w[0][grp], w[1][grp], 0x7632)};
        const uint32_t y[2] = {__byte_perm(w[2][grp], w[3][grp], 0x5410), __byte_perm(w[2][grp], w[3][grp], 0x7632)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // dims 64 grp + 16 i + g, + 8
            const uint32_t u = i & 1 ? x[i >> 1] >> 8 : x[i >> 1], z = i & 1 ? y[i >> 1] >> 8 : y[i >> 1];
            const uint32_t a0 = centred(u, false), a1 = centred(u, true), a2 = centred(z, false), a3 = centred(z, true);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816(o[n][4 * grp + i], a0, a1, a2, a3, b[n][0], b[n][1]);
        }
    }
}

#endif

}  // namespace remp
