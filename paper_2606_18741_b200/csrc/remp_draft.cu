// Verification of drafted tokens (rules: include/remp.h).
//
// Mathematics: a draft is accepted iff accept * q < p, which is exact in 64 bits for numbers of 32; the token behind the accepted ones is
// the first whose running sum of w = max(p - q, 0) (or of p) passes pick * (sum of all w). Sums are in 64 bits, in an order
// that depends on the vocabulary and the number of sequences alone.
//
// Bound: HBM, one or two vocabulary rows for each sequence; latency for few sequences. A sequence is a cluster of kBlocks thread
// blocks, a warp sums a stretch of consecutive tokens; the warps' sums are exchanged over distributed shared memory, and the
// warp whose stretch holds the token goes through it once more (it is in the caches).

#include <cooperative_groups.h>

#include <algorithm>

#include "remp_kv.h"

namespace remp {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32, kVec = 8;  // kVec: tokens of a lane at a time

struct DraftArgs {
    int32_t num_seqs, num_drafts, vocab;
    const int32_t *draft_start, *drafts;
    const uint8_t *target, *draft;
    int64_t s_target, s_draft;  // bytes
    const float *accept, *pick;
    int32_t *tokens, *accepted;
    uint32_t* error;
    int32_t wide;  // rows are 16-byte aligned
};

template <int kType>
__device__ __forceinline__ float value_of(const uint8_t* row, int i) {
    if constexpr (kType == REMP_DTYPE_FLOAT) return __ldg(reinterpret_cast<const float*>(row) + i);
    else if constexpr (kType == REMP_DTYPE_BFLOAT) return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(row) + i) << 16);
    else return __half2float(__ushort_as_half(__ldg(reinterpret_cast<const uint16_t*>(row) + i)));
}

// kVec tokens from i on; those from `end` on are 0.
template <int kType>
__device__ __forceinline__ void values_of(const uint8_t* row, int i, int end, bool wide, float (&x)[kVec]) {
    if (wide && i + kVec <= end) {
        if constexpr (kType == REMP_DTYPE_FLOAT) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(row + 4 * (int64_t)i)), b = __ldg(reinterpret_cast<const float4*>(row + 4 * (int64_t)i) + 1);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(row + 2 * (int64_t)i));
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (kType == REMP_DTYPE_BFLOAT) {
                    x[2 * k] = bf_low(w[k]), x[2 * k + 1] = bf_high(w[k]);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                    x[2 * k] = f.x, x[2 * k + 1] = f.y;
                }
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < kVec; ++k) x[k] = i + k < end ? value_of<kType>(row, i + k) : 0.f;
    }
}

struct Sums {  // of a warp's stretch
    double sum;
    int last;  // the last token with w > 0, or -1
};

struct Verdict {  // of all stretches: the sum, what the running sum has to pass, the sum before the stretch where it does
    double total, mark, before;
    int who, last;  // that stretch, or -1; the last token with w > 0
};

template <int kType, int kBlocks>
__global__ void __launch_bounds__(kThreads, 2) draft_verify_kernel(const __grid_constant__ DraftArgs a) {
    __shared__ Sums sums[2][kWarps];
    __shared__ Verdict verdict;
    __shared__ int shared_count;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int part = kBlocks > 1 ? (int)blockIdx.x % kBlocks : 0, s = blockIdx.x / kBlocks;
    const auto meet = [] {
        if constexpr (kBlocks > 1) cg::this_cluster().sync();
        else __syncthreads();
    };
    grid_begin();
    const int from = min(max(a.draft_start[s], 0), a.num_drafts), count = min(max(a.draft_start[s + 1], from), a.num_drafts) - from;
    if (part == 0 && tid == 0 && (from != a.draft_start[s] || from + count != a.draft_start[s + 1])) {
        if (a.error) atomicOr(a.error, (uint32_t)kErrBadLength);
    }
    const int64_t row0 = (int64_t)from + s;  // of target and tokens

    // ---- the accepted drafts: every block finds them for itself ----
    if (wid == 0) {
        int n = 0;
        for (; n < count; n += 32) {
            bool refused = false;
            if (n + lane < count) {
                const int64_t i = (int64_t)from + n + lane;
                const int x = a.drafts[i];
                refused = true;
                if (x >= 0 && x < a.vocab) {
                    const double p = value_of<kType>(a.target + (row0 + n + lane) * a.s_target, x);
                    const double q = a.draft ? (double)fmaxf(value_of<kType>(a.draft + i * a.s_draft, x), 0.f) : 1.0;
                    refused = !((double)a.accept[i] * q < p);
                } else if (part == 0 && a.error) {
                    atomicOr(a.error, (uint32_t)kErrBadLength);
                }
            }
            const unsigned votes = __ballot_sync(0xffffffffu, refused);
            if (votes) {
                n += __ffs(votes) - 1;
                break;
            }
        }
        if (lane == 0) shared_count = min(n, count);
    }
    __syncthreads();
    const int accepted = shared_count;
    const bool cut = accepted < count;
    if (part == 0) {
        for (int i = tid; i <= count; i += kThreads) {
            if (i < accepted) a.tokens[row0 + i] = a.drafts[from + i];
            else if (i > accepted) a.tokens[row0 + i] = -1;
        }
        if (tid == 0) a.accepted[s] = accepted;
    }

    // ---- the token behind them ----
    const uint8_t* p_row = a.target + (row0 + accepted) * a.s_target;
    const uint8_t* q_row = cut && a.draft ? a.draft + ((int64_t)from + accepted) * a.s_draft : nullptr;
    int without = cut && !a.draft ? a.drafts[from + accepted] : -1;
    constexpr int kStep = 32 * kVec;
    const int stretch = ((a.vocab + kBlocks * kWarps - 1) / (kBlocks * kWarps) + kStep - 1) / kStep * kStep;
    const int nth = part * kWarps + wid;
    const int begin = (int)min((int64_t)a.vocab, (int64_t)nth * stretch), end = (int)min((int64_t)a.vocab, (int64_t)begin + stretch);
    const auto doubles_of = [&](int i, double (&w)[kVec]) {
        float p[kVec], q[kVec];
        values_of<kType>(p_row, i, end, a.wide, p);
        if (q_row) values_of<kType>(q_row, i, end, a.wide, q);
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const double x = q_row ? (double)p[k] - fmaxf(q[k], 0.f) : (double)p[k];
            w[k] = x > 0. && i + k != without ? x : 0.;
        }
    };
    int turn = 0;
#pragma unroll 1
    for (;; turn = 1) {
        double sum = 0.;
        int last = -1;
#pragma unroll 2
        for (int i = begin + lane * kVec; i < end; i += kStep) {
            double w[kVec];
            doubles_of(i, w);
            sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
            for (int k = 0; k < kVec; ++k) last = w[k] > 0. ? i + k : last;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        last = __reduce_max_sync(0xffffffffu, last);
        if (lane == 0) sums[turn][wid] = Sums{sum, last};
        meet();
        // warp 0 of every block: sums before each warp's stretch, in order
        if (wid == 0) {
            constexpr int kAll = kBlocks * kWarps, kEach = kAll < 32 ? 1 : kAll / 32;  // consecutive stretches to a lane
            double mine[kEach], before[kEach], in = 0.;
            int lasts = -1;
#pragma unroll
            for (int x = 0; x < kEach; ++x) {
                const int w = lane * kEach + x;
                Sums y{0., -1};
                if (w < kAll) {
                    const Sums* of = &sums[turn][w % kWarps];
                    if constexpr (kBlocks > 1) of = cg::this_cluster().map_shared_rank(&sums[turn][w % kWarps], w / kWarps);
                    y = *of;
                }
                mine[x] = y.sum, before[x] = in, in += y.sum, lasts = max(lasts, y.last);
            }
            double upto = in;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const double up = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += up;
            }
            const double all = __shfl_sync(0xffffffffu, upto, 31), mark = (double)a.pick[s] * all, base = __shfl_up_sync(0xffffffffu, upto, 1);
            int found = -1;
            double found_before = 0.;
#pragma unroll
            for (int x = 0; x < kEach; ++x) {
                const double b = before[x] + (lane ? base : 0.);
                if (found < 0 && mine[x] > 0. && b + mine[x] > mark) found = lane * kEach + x, found_before = b;
            }
            const unsigned votes = __ballot_sync(0xffffffffu, found >= 0);
            const int src = votes ? __ffs(votes) - 1 : 0;
            found = __shfl_sync(0xffffffffu, found, src), found_before = __shfl_sync(0xffffffffu, found_before, src);
            lasts = __reduce_max_sync(0xffffffffu, lasts);
            if (lane == 0) verdict = Verdict{all, mark, found_before, found, lasts};
        }
        __syncthreads();
        if (verdict.total > 0. || turn || !cut) break;
        q_row = nullptr, without = -1;  // nothing is left of p - q: p
        __syncthreads();
    }
    __syncwarp();
    if constexpr (kBlocks > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");  // the others' sums are read
    // whose stretch holds it: the first whose running sum passes the mark; if none does, the last with a probability
    const double mark = verdict.mark, before = verdict.before;
    const int who = verdict.who, fallback = verdict.last;
    if (who < 0) {
        if (part == 0 && tid == 0) {
            a.tokens[row0 + accepted] = fallback;
            if (fallback < 0 && a.error) atomicOr(a.error, (uint32_t)kErrOverflow);
        }
    } else if (nth == who) {
        // lane by lane of its steps, several side by side; then token by token of the one lane where the sum passes
        constexpr int kAtOnce = 4;
        double sum = before;
        int token = sums[turn][wid].last;
        bool done = false;
#pragma unroll 1
        for (int i0 = begin; i0 < end && !done; i0 += kAtOnce * kStep) {
            double mine[kAtOnce], in[kAtOnce];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                double w[kVec];
                doubles_of(min(i0 + x * kStep + lane * kVec, end), w);
                in[x] = mine[x] = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1)
#pragma unroll
                for (int x = 0; x < kAtOnce; ++x) {
                    const double up = __shfl_up_sync(0xffffffffu, in[x], d);
                    if (lane >= d) in[x] += up;
                }
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const unsigned votes = done ? 0 : __ballot_sync(0xffffffffu, mine[x] > 0. && sum + in[x] > mark);
                if (votes) {
                    const int src = __ffs(votes) - 1, i = i0 + x * kStep + src * kVec;
                    double at = __shfl_sync(0xffffffffu, sum + (in[x] - mine[x]), src), w[kVec];
                    doubles_of(i, w);
                    int last = -1, found = -1;
#pragma unroll
                    for (int k = 0; k < kVec; ++k) {
                        at += w[k];
                        if (w[k] > 0.) last = i + k;
                        if (found < 0 && w[k] > 0. && at > mark) found = i + k;
                    }
                    token = found >= 0 ? found : last, done = true;
                }
                sum += __shfl_sync(0xffffffffu, in[x], 31);
            }
        }
        if (lane == 0) a.tokens[row0 + accepted] = token;
    }
    __syncwarp();
    if constexpr (kBlocks > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // nobody leaves while its sums are read
}

template <int kType>
cudaError_t launch(const DraftArgs& a, int sms, cudaStream_t stream) {
    // Long rows: as many blocks for a sequence as fit the GPU at two to an SM. 64 sequences of 131072 tokens: 19 us with 4, 23 us
    // with 8.
    const int64_t room = 2 * sms / a.num_seqs;
    if (a.vocab <= 8192 || room < 2) return launch_after(draft_verify_kernel<kType, 1>, a.num_seqs, kThreads, 0, stream, a);
    if (room < 4) return launch_after_in_clusters(draft_verify_kernel<kType, 2>, (int64_t)a.num_seqs * 2, 2, kThreads, 0, stream, a);
    if (room < 8) return launch_after_in_clusters(draft_verify_kernel<kType, 4>, (int64_t)a.num_seqs * 4, 4, kThreads, 0, stream, a);
    return launch_after_in_clusters(draft_verify_kernel<kType, 8>, (int64_t)a.num_seqs * 8, 8, kThreads, 0, stream, a);
}

}  // namespace

}  // namespace remp

using namespace remp;

extern "C" remp_status remp_draft_verify(int32_t num_seqs, int32_t num_drafts, int32_t vocab, const int32_t* draft_start,
                                         const int32_t* drafts, const void* target, int64_t target_stride, const void* draft_probs,
                                         int64_t draft_stride, int32_t dtype, const float* accept, const float* pick, int32_t* tokens,
                                         int32_t* accepted, uint32_t* error, void* stream_) {
    if (num_seqs < 0 || num_drafts < 0 || vocab < 1) return fail(REMP_ERR_INVALID_ARG, "negative number of sequences or drafts, or no vocabulary");
    if (dtype != REMP_DTYPE_BFLOAT && dtype != REMP_DTYPE_HALF && dtype != REMP_DTYPE_FLOAT) return fail(REMP_ERR_INVALID_ARG, "unknown dtype");
    if (vocab > 1 << 30 || num_seqs > 0x7fffffff / 16 || num_drafts > 0x7fffffff - num_seqs) return fail(REMP_ERR_SHAPE, "too many tokens, sequences or drafts");
    if (num_seqs == 0) return REMP_OK;
    if (!draft_start || !target || !pick || !tokens || !accepted || (num_drafts > 0 && (!drafts || !accept)))
        return fail(REMP_ERR_INVALID_ARG, "null argument");
    const int64_t size = dtype == REMP_DTYPE_FLOAT ? 4 : 2;
    if ((num_seqs + num_drafts > 1 && target_stride < vocab) || (draft_probs && num_drafts > 1 && draft_stride < vocab))
        return fail(REMP_ERR_SHAPE, "rows of probabilities overlap");
    if ((reinterpret_cast<uint64_t>(target) | reinterpret_cast<uint64_t>(draft_probs)) & (size - 1))
        return fail(REMP_ERR_SHAPE, "probabilities must be aligned to their type");
    DraftArgs a{num_seqs, num_drafts, vocab, draft_start, drafts, static_cast<const uint8_t*>(target), static_cast<const uint8_t*>(draft_probs),
                target_stride * size, draft_probs ? draft_stride * size : 0, accept, pick, tokens, accepted, error, 0};
    a.wide = !((reinterpret_cast<uint64_t>(target) | reinterpret_cast<uint64_t>(draft_probs) | (uint64_t)a.s_target | (uint64_t)a.s_draft) & 15);
    int device = -1, sms = 0;
    REMP_CUDA(cudaGetDevice(&device));
    REMP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    REMP_CUDA(dtype == REMP_DTYPE_FLOAT ? launch<REMP_DTYPE_FLOAT>(a, sms, stream)
              : dtype == REMP_DTYPE_BFLOAT ? launch<REMP_DTYPE_BFLOAT>(a, sms, stream) : launch<REMP_DTYPE_HALF>(a, sms, stream));
    return REMP_OK;
}
