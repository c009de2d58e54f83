// Pieces of attention over a tile of 16 tokens of the 4-bit cache, one warp: fetch, queries, scores, values.
// Lane (g, t) = (lane / 4, lane % 4), as the matrix instructions number rows and columns.
#pragma once

#include <algorithm>

#include "remp_kvq.h"

namespace remp {

constexpr int kAttendMaxCtas = 512;
constexpr size_t kAttendCounterBytes = kAttendMaxCtas * 4;
constexpr size_t kAttendWorkspace = kAttendCounterBytes + (size_t)2 * kAttendMaxCtas * 16 * (128 + 2) * 4;

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

// A tile of K (at `src`) and its tile of V (`kv` bytes behind) to shared memory, 16 bytes at a time. The pieces of V's
// codes change places within 128 bytes (piece ^ (token & 6)), so that the lanes of a warp, which read four tokens' rows
// at once, meet different banks.
template <int D>
__device__ __forceinline__ void kvq_fetch_tile(const uint8_t* src, int64_t kv, uint32_t dst, int lane) {
    constexpr int kBytes = kKvqTile * kvq_token_bytes(D), kPieces = kBytes / 16, kCodes = kKvqTile * D / 32;
    const uint8_t* k = src + lane * 16;
    const uint8_t* v = k + kv - kBytes;  // piece p of both tiles is at v + 16 * (p - lane) once p >= kPieces
#pragma unroll
    for (int i = 0; i < (2 * kPieces + 31) / 32; ++i) {
        const int p = lane + 32 * i;
        if (32 * i + 31 < kPieces) {
            cp_async16(dst + p * 16, k + 512 * i);
        } else {
            const int pv = p - kPieces;
            const int to = (32 * i >= kPieces || pv >= 0) && pv < kCodes ? pv ^ ((pv / (D / 32)) & 6) : pv;
            if (32 * i + 31 < 2 * kPieces || p < 2 * kPieces)
                cp_async16(dst + kBytes + to * 16, (32 * i >= kPieces || pv >= 0 ? v : k) + 512 * i);
        }
    }
}

// The operand columns of one row of queries (src points at dim 2t). Slots 0..7 of each 16 dims are taken 16-fold: they
// meet codes at bits 0..3, the others codes at bits 4..7. A power of two brings the row's largest value to [8, 16), so that
// halves hold 16-bit queries of any size exactly (down to 2^-28 of the largest). qsum: 2^-20 times the sums of
// the groups, and back: what a score is multiplied with, both for columns 2t and 2t+1.
template <int D>
__device__ __forceinline__ void kvq_load_queries(const uint16_t* src, bool bf, bool real, int t, uint32_t (&qf)[D / 16][2],
                                                 float (&qsum)[D / kKvqGroup][2], float (&back)[2], float scale_log2) {
    uint32_t raw[D / 16][2];
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) raw[i][h] = real ? *reinterpret_cast<const uint32_t*>(src + 16 * i + 8 * h) : 0u;
    const auto value = [&](uint32_t w) {
        return bf ? make_float2(bf_low(w), bf_high(w)) : __half22float2(*reinterpret_cast<const __half2*>(&w));
    };
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float2 f = value(raw[i][h]);
            top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^e with top * 2^e in [8, 16); 0, infinities and rows below 2^-90 keep a bounded exponent
    const int exponent = (int)(__float_as_uint(top) >> 23) - 127;
    const int e = top > 0.f ? max(-120, min(93, 3 - exponent)) : 0;
    const float up = __uint_as_float((uint32_t)(127 + e) << 23);
    const float down = scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23);
    float sums[D / kKvqGroup];
#pragma unroll
    for (int i = 0; i < D / kKvqGroup; ++i) sums[i] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float2 f = value(raw[i][h]);
            f.x *= up, f.y *= up;
            sums[i / 4] += f.x + f.y;
            const float times = h ? 1.f : 16.f;
            qf[i][h] = pack2(f.x * times, f.y * times, false);
        }
#pragma unroll
    for (int i = 0; i < D / kKvqGroup; ++i) {
        sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], 1);
        sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], 2);
        sums[i] *= 9.5367431640625e-7f;  // 2^-20, as the products with codes
#pragma unroll
        for (int c = 0; c < 2; ++c) qsum[i][c] = __shfl_sync(0xffffffffu, sums[i], (2 * t + c) * 4);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) back[c] = __shfl_sync(0xffffffffu, down * 1048576.f, (2 * t + c) * 4);
}

// The steps and minima of tokens g (h = 0) and g+8 of a tile, one word for each group.
template <int D>
__device__ __forceinline__ void kvq_params(const uint8_t* tile, int g, uint32_t (&par)[2][D / kKvqGroup]) {
    constexpr int G = D / kKvqGroup;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint8_t* p = tile + kKvqTile * D / 2 + (g + 8 * h) * (D / 16);
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
__device__ __forceinline__ void kvq_scores(const uint8_t* tile, int g, int t, const uint32_t (&qf)[NT][D / 16][2],
                                           const float (&qsum)[NT][D / kKvqGroup][2], float (&s)[NT][4]) {
    constexpr int G = D / kKvqGroup, W = D / 32;  // groups, words of a lane's row
    uint32_t w[2][W], par[2][G];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint8_t* row = tile + (g + 8 * h) * (D / 2) + t * (D / 8);
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
    kvq_params<D>(tile, g, par);
#pragma unroll
    for (int grp = 0; grp < G; ++grp) {
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
#pragma unroll
        for (int i = 2 * grp; i < 2 * grp + 2; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // dims 32i + 16h .. +15
                const uint32_t x0 = h ? w[0][i] >> 8 : w[0][i], x1 = h ? w[1][i] >> 8 : w[1][i];
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    mma16816(acc[n], x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u,
                             qf[n][2 * i + h][0], qf[n][2 * i + h][1]);
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
    const uint32_t y = (x & (upper ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&y), __half2half2(__ushort_as_half(upper ? 0x6480 : 0x6408)));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// o += (V's codes - 8)^T . R^T (16-fold in rows g+8 of each 16 dims), where R = p * step rounded to half; low += sums of
// p * (minimum + 8 step); so sum p*v = o + low. Codes around 0 keep the sums of a long sequence small: the matrix
// instructions' sums are cut, not rounded, and over 100 thousand tokens codes of one sign put the result off by 2^-18
// of sum p*v's terms; what rounding R does is halved as well. p: the probabilities in kvq_scores' layout; par: kvq_params of the tile, 0
// for tokens that are not there.
template <int D, int NT>
__device__ __forceinline__ void kvq_values(const uint8_t* tile, int g, int t, const float (&p)[NT][4],
                                           const uint32_t (&par)[2][D / kKvqGroup], float (&o)[NT][D / 16][4],
                                           float (&low)[NT][D / kKvqGroup][2]) {
    constexpr int G = D / kKvqGroup;
    uint32_t w[4][G];  // tokens 2t, 2t+1, 2t+8, 2t+9: this lane's dims of each group
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = ((2 * t + (j & 1) + (j >> 1) * 8) * (D / 2) + g * (D / 16)) ^ ((2 * t) << 4);
        if constexpr (G == 1) {
            w[j][0] = *reinterpret_cast<const uint32_t*>(tile + at);
        } else if constexpr (G == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(tile + at);
            w[j][0] = x.x, w[j][1] = x.y;
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(tile + at);
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
