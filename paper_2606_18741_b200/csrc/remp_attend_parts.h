// Attention whose work is cut evenly over the warps of a grid: a warp's share begins and ends inside a unit (rows of a
// sequence and a KV head), and the parts of a unit are merged in the order of the list. For kernels that hold the output as
// O^T, 16 dims by 8 rows to a matrix instruction: lane (g, t) = (lane / 4, lane % 4) has dims 16i + g, 16i + 8 + g of rows 8n + 2t, +1.
#pragma once

#include "remp_kvq_device.h"

namespace remp {

#ifdef __CUDACC__

// Args: what a kernel of this kind takes; has out, lse, q_heads, group, by_group and workspace.
template <class Args>
__device__ __forceinline__ int token_of(const Args& a, int row) { return a.by_group ? (int)__umulhi((uint32_t)row, a.by_group) : row; }

constexpr float kNoRef = -3e38f;  // reference of a row that has seen nothing; finite, so that -inf - kNoRef is -inf

struct Unit {  // rows [row0, row0 + rows) of a sequence (first row of the batch q0) and a KV head; its steps in the list
    int from, to;
    int q0, row0, rows, head;
    int live;
};

struct Chain {  // parts of one unit in the order of the list: the first, and from rest + stride on; merged into slot or the output
    const float *first, *rest;
    float* slot;
    int64_t stride;
    const Unit* unit;
    int n;
};

// One quad of results: dims 16i + g, 16i + 8 + g of columns 8n + 2t, +1 -> the output, 4 bytes to a lane.
template <bool BF>
__device__ __forceinline__ void put_quad(const float4& o, const float (&inv)[2], uint16_t* dst, bool real) {
    const uint32_t x = transpose8(pack2(o.x * inv[0], o.y * inv[1], BF)), y = transpose8(pack2(o.z * inv[0], o.w * inv[1], BF));
    if (real) *reinterpret_cast<uint32_t*>(dst) = x, *reinterpret_cast<uint32_t*>(dst + 8) = y;
}

// Where row 8n + g of a unit goes (dim 2t of it).
template <class Args>
__device__ __forceinline__ uint16_t* out_row(const Args& a, const Unit& u, int n, int g, int t) {
    const int r = u.row0 + 8 * n + g, token = token_of(a, r);
    return a.out.data + (int64_t)(u.q0 + token) * a.out.s_token + (int64_t)(u.head * a.group + r - token * a.group) * a.out.s_head + 2 * t;
}

template <class Args>
__device__ __forceinline__ void put_lse(const Args& a, const Unit& u, int col, float ref, float sum) {
    const int r = u.row0 + col, token = token_of(a, r);
    if (col < u.rows)
        a.lse[(int64_t)(u.q0 + token) * a.q_heads + u.head * a.group + r - token * a.group] =
            sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
}

// Parts are read in shared memory or, written by other blocks, in global memory: past the first-level cache.
__device__ __forceinline__ float4 part4(const float* p) {
    float4 x;
    asm volatile("ld.volatile.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "l"(p));
    return x;
}
__device__ __forceinline__ float2 part2(const float* p) {
    float2 x;
    asm volatile("ld.volatile.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "l"(p));
    return x;
}

// Quad q of a chain.
template <class Z, bool BF, class Args>
__device__ __forceinline__ void merge_quad(const Args& a, const Chain& c, int q, int lane) {
    constexpr int D = Z::kDim;
    const int g = lane >> 2, t = lane & 3, tile = q / (D / 16), col = 8 * tile + 2 * t;
    float2 ref = make_float2(kNoRef, kNoRef), sum = make_float2(0.f, 0.f);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAhead = 8;
#pragma unroll 1
    for (int i0 = 0; i0 < c.n; i0 += kAhead) {
        float4 o[kAhead];
        float2 r[kAhead], s[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const float* x = i0 + j ? c.rest + (i0 + j) * c.stride : c.first;
            r[j] = make_float2(kNoRef, kNoRef), s[j] = make_float2(0.f, 0.f), o[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i0 + j < c.n) o[j] = part4(x + q * 128 + lane * 4), r[j] = part2(x + Z::kQuads * 128 + col), s[j] = part2(x + Z::kQuads * 128 + Z::kRows + col);
        }
        float2 top = ref;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) top.x = fmaxf(top.x, r[j].x), top.y = fmaxf(top.y, r[j].y);
        float fx = exp2_approx(ref.x - top.x), fy = exp2_approx(ref.y - top.y);
        sum.x *= fx, sum.y *= fy, acc.x *= fx, acc.y *= fy, acc.z *= fx, acc.w *= fy;
        ref = top;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + j >= c.n) break;
            fx = exp2_approx(r[j].x - top.x), fy = exp2_approx(r[j].y - top.y);
            sum.x = fmaf(fx, s[j].x, sum.x), sum.y = fmaf(fy, s[j].y, sum.y);
            acc.x = fmaf(fx, o[j].x, acc.x), acc.y = fmaf(fy, o[j].y, acc.y);
            acc.z = fmaf(fx, o[j].z, acc.z), acc.w = fmaf(fy, o[j].w, acc.w);
        }
    }
    const bool keeper = q % (D / 16) == 0 && g == 0;  // of the rows' references and sums
    if (c.slot) {
        *reinterpret_cast<float4*>(c.slot + q * 128 + lane * 4) = acc;
        if (keeper) {
            *reinterpret_cast<float2*>(c.slot + Z::kQuads * 128 + col) = ref;
            *reinterpret_cast<float2*>(c.slot + Z::kQuads * 128 + Z::kRows + col) = sum;
        }
    } else {
        const Unit u = *c.unit;
        const float inv[2] = {sum.x == 0.f ? 0.f : 1.f / sum.x, sum.y == 0.f ? 0.f : 1.f / sum.y};
        put_quad<BF>(acc, inv, out_row(a, u, tile, g, t) + q % (D / 16) * 16, 8 * tile + g < u.rows);
        if (keeper && a.lse) put_lse(a, u, col, ref.x, sum.x), put_lse(a, u, col + 1, ref.y, sum.y);
    }
}

// Behind a kernel's list: parts[w] are the unit that warp w found begun and the one that it left unfinished, in the second and the first
// place of its shared memory (Z::kRing, 0). [cta0, cta1): this block's places in the list, `per` a block's. Z: kDim, kRows,
// kQuads, kPartFloats, kRing, kWarpBytes, kWarps.
template <class Z, bool BF, class Args>
__device__ __forceinline__ void merge_parts(const Args& a, uint8_t* smem, Unit (*parts)[2], Chain* chains, int* num_chains, const int cta0, const int cta1,
                                            const int per) {
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    // ---- parts of one unit: first those in this block, then those of several blocks, by the block that arrives last ----
    uint32_t* counters = reinterpret_cast<uint32_t*>(a.workspace);
    float* slots = reinterpret_cast<float*>(a.workspace + kAttendCounterBytes);
    bool shared = false;  // thread's chain is of a unit that other blocks have parts of
    Chain c{};
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
        __syncthreads();
        if (wid == 0) {
            if (round == 0 && lane <= Z::kWarps) {
                // chains begin with the part that an earlier block began (lane 0), or with a warp's tail
                const int at = max(lane - 1, 0);
                const Unit* u = &parts[at][lane > 0];
                if (u->live) {
                    c.n = 1;
#pragma unroll 1
                    while (at + c.n < Z::kWarps && parts[at + c.n][0].live && parts[at + c.n][0].from == u->from) ++c.n;
                    uint8_t* warp = smem + at * Z::kWarpBytes;
                    c.rest = reinterpret_cast<const float*>(warp + Z::kRing), c.first = lane > 0 ? reinterpret_cast<const float*>(warp) : c.rest;
                    c.stride = Z::kWarpBytes / 4, c.unit = u;
                    shared = u->from < cta0 || u->to > cta1;
                    if (shared) c.slot = slots + (2 * blockIdx.x + (u->from >= cta0)) * Z::kPartFloats;
                }
            } else if (round == 1) {
                c.n = 0;
                if (shared) {
                    const int first = (int)((uint32_t)c.unit->from / (uint32_t)per), last = (int)((uint32_t)(c.unit->to - 1) / (uint32_t)per);
                    uint32_t before;
                    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(counters + first) : "memory");
                    if (before == (uint32_t)(last - first)) {
                        counters[first] = 0;  // ready for the next call
                        c.first = slots + (2 * first + 1) * Z::kPartFloats, c.rest = c.first - Z::kPartFloats, c.stride = 2 * Z::kPartFloats;
                        c.slot = nullptr, c.n = last - first + 1;
                    }
                }
            }
            const unsigned live = __ballot_sync(0xffffffffu, c.n > 0);
            if (c.n > 0) chains[__popc(live & ((1u << lane) - 1))] = c;
            if (lane == 0) *num_chains = __popc(live);
        }
        const bool any = __syncthreads_or(shared);
        const int tasks = *num_chains * Z::kQuads;
#pragma unroll 1
        for (int task = wid; task < tasks; task += Z::kWarps) merge_quad<Z, BF>(a, chains[task / Z::kQuads], task % Z::kQuads, lane);
        if (!any) return;
    }
}

#endif

}  // namespace remp
