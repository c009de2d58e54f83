// The weight that attention gives to cached positions, for many rows of a sequence (rules: include/remp.h).
//
// Mathematics: weight of key j += sum over rows r that see it of 2^(q_r.k_j * scale - lse_r), scale and lse in powers of two. With
// S^T = K.Q^T, 128 keys by up to 256 rows, a key is a lane of the tensor memory: one thread adds up a key's row in registers, and
// nothing crosses lanes. More rows take further rounds over the same keys, each added by the thread that wrote the last.
// Rounding: scores, probabilities and sums are in 32 bits; nothing is rounded to fewer.
//
// Bound: the exponentials (one for each row and key, 16 a cycle of an SM; the products of 128 dims take half as long). A thread
// block takes a range of the keys of one sequence and KV head. Eight warps weigh, four for the even chunks of 32 rows and four for
// the odd ones; one thread issues the matrix instructions, a block of keys ahead (two buffers of S^T); one warp brings K through a
// ring. The rows that see a key are a range of them, so a mask is two numbers for each key and round. 2 x 32 queries of 32 heads over
// 16383 tokens of 4 KV heads, 128 dims: 23 us, 93 in the kernel for few rows.
//
// Every wait is on a barrier in shared memory and bounded. A block that gives up goes on without waiting, writes NaN and sets
// error bit 4; it leaves when all that it has asked for is done.

#include "remp_kv_boxes.h"
#include "remp_kv_weigh.h"
#include "remp_kvq_device.h"

namespace remp {

namespace {

constexpr int kKeys = 128, kMostSplits = 512, kWeighWarps = 8, kThreads = (kWeighWarps + 2) * 32;

template <int D>
struct Wide {
    static constexpr int kRows = D == 256 ? 128 : 256;                  // of a round: Q of them lies beside the ring
    static constexpr int kQ = kRows * D * 2, kItem = kKeys * D * 2, kEight = 8 * D * 2;
    static constexpr int kPlaces = D == 256 ? 2 : 4;                    // of the ring
    static constexpr int kBytes = kQ + kPlaces * kItem + 1024;
};

struct WideArgs {
    KvBoxes boxes;
    WeighArgs w;
    int32_t splits, tries;  // ranges of the keys of a sequence and head; of the wait for the queries
};

template <int D, bool BF>
__global__ void __launch_bounds__(kThreads, 1) kv_weigh_wide_kernel(const __grid_constant__ WideArgs p_) {
    using Z = Wide<D>;
    constexpr uint32_t kType = BF ? kShapeBfloat : 0;
    constexpr int kPlaces = Z::kPlaces;
    const WeighArgs& a = p_.w;
    const KvView& v = a.v;
    extern __shared__ uint8_t smem_[];
    __shared__ __align__(8) uint64_t bars[6 + 2 * kPlaces];
    __shared__ __align__(16) float norms[Z::kRows];  // of a round's rows: -lse in powers of two, -infinity for rows that count nothing
    __shared__ float halves[2][kKeys];
    __shared__ __align__(8) uint8_t gone[8][8];      // of a block of keys: tiles that are not there, or that no row sees
    __shared__ uint32_t tmem_at;
    __shared__ int dead, silent;                     // the block has given up; the round in which rows were met that count nothing
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    grid_begin();

    // ---- this block's keys ----
    const int unit = blockIdx.x / p_.splits, split = blockIdx.x - unit * p_.splits, seq = unit / v.kv_heads, head = unit - seq * v.kv_heads;
    const KvqSpan span = kvq_span(v.query_start[seq], v.query_start[seq + 1], v.seq_lens[seq], v.num_tokens, a.room);
    if (kvq_span_bad(span, v.seq_lens[seq]) && head == 0 && split == 0 && tid == 0) kvq_error(v, kErrBadLength);
    const int rows_all = span.queries * a.group, rounds = (rows_all + Z::kRows - 1) / Z::kRows, len = span.len, first_pos = span.first_pos;
    // all of them when every position is written, else those of the first tokens, then those of the window
    const int low_from = a.fresh ? 0 : kvq_first_key(first_pos, a.window);
    int begin = min(len, low_from) / kKvqTile * kKvqTile, ahead = (min(min(a.first, len), begin) + kKeys - 1) / kKeys;
    if (ahead * kKeys >= begin) begin = ahead = 0;
    const int blocks_all = ahead + (len - begin + kKeys - 1) / kKeys;
    const int b0 = (int)((long long)blocks_all * split / p_.splits), blocks = (int)((long long)blocks_all * (split + 1) / p_.splits) - b0;
    if (rows_all == 0 || blocks == 0) return;
    const auto key_of = [&](int j) { return b0 + j < ahead ? (b0 + j) * kKeys : begin + (b0 + j - ahead) * kKeys; };  // the first key of block j
    const int items = blocks * rounds;

    uint8_t* smem = smem_ + ((1024u - ((uint32_t)__cvta_generic_to_shared(smem_) & 1023u)) & 1023u);
    uint8_t *sq = smem, *ring = smem + Z::kQ;
    // scores there, scores read, of each buffer; queries of a round; places of the ring
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars), s_full = bar, s_free = bar + 16, q_full = bar + 32, all_done = bar + 40, full = bar + 48, vacant = full + 8 * kPlaces;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) bar_init(s_full + 8 * i, 1), bar_init(s_free + 8 * i, kWeighWarps);
        for (int i = 0; i < kPlaces; ++i) bar_init(full + 8 * i, 1), bar_init(vacant + 8 * i, 1);
        bar_init(q_full, 1), bar_init(all_done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead = 0, silent = -1;
        for (int i = 0; i < 8; ++i) *reinterpret_cast<unsigned long long*>(gone[i]) = 0;
    }
    if (wid == kWeighWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_at)),
                     "n"(2 * Z::kRows)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = tmem_at;
    const auto chunks_of = [&](int round) { return (min(Z::kRows, rows_all - round * Z::kRows) + 31) / 32; };  // of 32 rows

    if (wid < kWeighWarps) {
        const int part = wid >> 2, mine = tid & 127;  // chunks part, part + 2, ..; the key in its block
        const uint32_t lanes = tmem + ((uint32_t)((wid & 3) * 32) << 16);
        float* const weights = a.weights + ((int64_t)seq * v.kv_heads + head) * a.stride;
        int item = 0;
#pragma unroll 1
        for (int round = 0; round < rounds; ++round) {
            // ---- the round's queries; the scores of the last one are all read, so its queries are too ----
            const int row0 = round * Z::kRows, rows = min(Z::kRows, rows_all - row0), chunks = chunks_of(round);
            asm volatile("bar.sync 1, %0;" ::"n"(kWeighWarps * 32) : "memory");
            constexpr int kPieces = D / 8;
#pragma unroll 4
            for (int i = tid; i < chunks * 32 * kPieces; i += kWeighWarps * 32) {
                const int r = i / kPieces, piece = i % kPieces, row = row0 + min(r, rows - 1), token = kv_token_of(a.by_group, row);
                uint4 x = *reinterpret_cast<const uint4*>(a.q.data + (int64_t)(span.q0 + token) * a.q.s_token + (int64_t)(head * a.group + row - token * a.group) * a.q.s_head + 8 * piece);
                if (r >= rows) x = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(sq + (piece / 8) * (Z::kRows * 128) + r * 128 + (((piece % 8) ^ (r & 7)) << 4)) = x;
            }
            if (tid < chunks * 32) {
                float norm = -INFINITY;
                if (tid < rows) {
                    const int row = row0 + tid, token = kv_token_of(a.by_group, row);
                    const float l = __ldg(a.lse + (int64_t)(span.q0 + token) * a.q_heads + head * a.group + row - token * a.group);
                    if (l == -INFINITY) silent = round;
                    else norm = l * -1.4426950408889634f;
                }
                norms[tid] = norm;
            }
            for_tensor_cores();
            asm volatile("bar.sync 1, %0;" ::"n"(kWeighWarps * 32) : "memory");
            if (tid == 0) bar_arrive(q_full);
            const bool all_count = *static_cast<volatile int*>(&silent) != round;
            const int low = first_pos + kv_token_of(a.by_group, row0), high = first_pos + kv_token_of(a.by_group, row0 + rows - 1);  // positions of the first and last row
            const int high_from = kvq_first_key(high, a.window);

            // ---- keys: one to a thread of each half of the warps ----
#pragma unroll 1
            for (int j = 0; j < blocks; ++j, ++item) {
                const int buffer = item & 1, key0 = key_of(j), key = key0 + mine;
                bar_wait(s_full + 8 * buffer, item >> 1 & 1, &dead);
                __syncwarp();
                tmem_after();
                const unsigned long long missing = *reinterpret_cast<const volatile unsigned long long*>(gone[item & 7]);
                const bool whole = all_count && missing == 0 && key0 + kKeys - 1 <= low && (key0 >= high_from || key0 + kKeys <= a.first);
                // rows [from, from + count) of the round see this key
                int from = 0, count = whole ? rows : 0;
                if (!whole && !(missing >> (8 * (mine / kKvqTile)) & 1)) {
                    const long long least = max(0LL, (long long)key - first_pos), most = a.window > 0 && key >= a.first ? (long long)key + a.window - first_pos : rows_all;
                    const long long r0 = max(0LL, least * a.group - row0), r1 = min((long long)rows, most * a.group - row0);
                    if (r1 > r0) from = (int)r0, count = (int)(r1 - r0);
                }
                float2 sum[2] = {};
#pragma unroll 1
                for (int c = part; c < chunks; c += 2) {
                    uint32_t s[32];
                    tmem_ask32(lanes + buffer * Z::kRows + 32 * c, s);
                    tmem_there32(s);
                    if (whole && 32 * c + 32 <= rows) {
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float4 n = *reinterpret_cast<const float4*>(norms + 32 * c + 2 * i);
                            float2 x = fma2(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), make_float2(a.scale_log2, a.scale_log2), make_float2(n.x, n.y));
                            float2 y = fma2(make_float2(__uint_as_float(s[2 * i + 2]), __uint_as_float(s[2 * i + 3])), make_float2(a.scale_log2, a.scale_log2), make_float2(n.z, n.w));
                            x.x = exp2_approx(x.x), x.y = exp2_approx(x.y), y.x = exp2_approx(y.x), y.y = exp2_approx(y.y);
                            sum[0] = add2(sum[0], x), sum[1] = add2(sum[1], y);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float n = norms[32 * c + i], x = exp2_approx(fmaf(__uint_as_float(s[i]), a.scale_log2, n));
                            sum[0].x += (uint32_t)(32 * c + i - from) < (uint32_t)count && n != -INFINITY ? x : 0.f;
                        }
                    }
                }
                tmem_before();
                __syncwarp();
                if (lane == 0) bar_arrive(s_free + 8 * buffer);
                const float2 both = add2(sum[0], sum[1]);
                const float half = both.x + both.y;
                // the halves meet, warp by warp
                if (part == 1) halves[buffer][mine] = half;
                asm volatile("bar.sync %0, 64;" ::"r"(2 + (wid & 3)) : "memory");
                if (part == 0 && key < len) {
                    float x = half + halves[buffer][mine];
                    if (*static_cast<volatile int*>(&dead)) x = __uint_as_float(0x7fc00000u);
                    weights[key] = round == 0 && (a.fresh || key >= first_pos) ? x : weights[key] + x;
                }
            }
        }
    } else if (wid == kWeighWarps) {
        // ---- matrix instructions: one thread waits and issues ----
        if (elect_one()) {
            const uint64_t q_at = operand_at((uint32_t)__cvta_generic_to_shared(sq)), ring_at = operand_at((uint32_t)__cvta_generic_to_shared(ring)) + keys_apart(Z::kEight);
            int item = 0;
#pragma unroll 1
            for (int round = 0; round < rounds; ++round) {
                const uint32_t shape = shape_of(0) + ((uint32_t)chunks_of(round) << 19) | kType;  // 32 columns for each chunk
                bar_wait(q_full, round & 1, &dead, p_.tries);
#pragma unroll 1
                for (int j = 0; j < blocks; ++j, ++item) {
                    const int place = item % kPlaces, buffer = item & 1;
                    bar_wait(full + 8 * place, item / kPlaces & 1, &dead);
                    if (item > 1) bar_wait(s_free + 8 * buffer, (item >> 1) - 1 & 1, &dead);
                    tmem_after();
                    const uint64_t k_at = ring_at + (uint32_t)(place * (Z::kItem >> 4));
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_smem_one(tmem + buffer * Z::kRows, k_at + ((k / 4) * 1024 + (k % 4) * 32 >> 4), q_at + ((k / 4) * (Z::kRows * 128) + (k % 4) * 32 >> 4), shape, k > 0);
                    commit_one(s_full + 8 * buffer), commit_one(vacant + 8 * place);
                }
            }
            // nothing stays in flight: a barrier of its own behind everything, then the last arrival on each of these
            commit_one(all_done);
            bar_drain(all_done, 1, &dead);
            for (int i = 0; i < 2; ++i) bar_drain(s_full + 8 * i, (items + 1 - i) / 2, &dead);
            for (int i = 0; i < kPlaces; ++i) bar_drain(vacant + 8 * i, (items - i + kPlaces - 1) / kPlaces, &dead);
        }
        __syncwarp();
    } else {
        // ---- keys: a tile to a lane; what a slot behind the length holds is its own lane's business ----
        constexpr int kTiles = kKeys / kKvqTile;
        const int32_t* row = v.tables + (int64_t)seq * v.max_blocks;
        const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
        // Whether a row sees something of the tile from `key` on; others are not looked up: their pages may have been given back.
        const int seen_from = kvq_first_key(first_pos, a.window);
        const auto wanted = [&](int key) { return lane < kTiles && key < len && (key + kKvqTile > seen_from || key < a.first); };
        const auto find = [&](int j) {  // this lane's tile of block j: its block (-1: not asked for) and first token in it
            int2 r = make_int2(-1, 0);
            const int key = key_of(j) + lane * kKvqTile;
            if (wanted(key)) {
                const int tile = key / kKvqTile, in_row = tile / v.block_tiles;
                r = make_int2(__ldg(row + in_row), (tile - in_row * v.block_tiles) * kKvqTile);
            }
            return r;
        };
        int2 next = find(0);
        int item = 0, j = 0;
#pragma unroll 1
        for (; item < items; ++item) {
            const int place = item % kPlaces, turn = item / kPlaces, key = key_of(j) + lane * kKvqTile;
            const int2 at = next;
            if (++j == blocks) j = 0;
            next = find(j);
            const bool there = (uint32_t)at.x < (uint32_t)v.nb;
            if (!there && wanted(key)) kvq_error(v, kErrBadBlock);
            if (turn > 0) bar_wait(vacant + 8 * place, (turn - 1) & 1, &dead);
            if (__any_sync(0xffffffffu, *static_cast<volatile int*>(&dead))) break;  // what is asked for is waited for below
            if (lane < kTiles) gone[item & 7][lane] = !there;
            const uint32_t boxes = __ballot_sync(0xffffffffu, there);
            __syncwarp();  // all lanes' marks before the arrival that tells of them: a vote orders no memory
            if (lane == 0) bar_arrive_expecting(full + 8 * place, __popc(boxes) * (kKvqTile * D * 2));
            __syncwarp();
            if (there) bring_tile(ring_at + place * Z::kItem + lane * (2 * Z::kEight), &p_.boxes.k, full + 8 * place, at.y / 8, at.x * p_.boxes.i_block + head * p_.boxes.i_head);
        }
        __syncwarp();
        for (int i = 0; i < kPlaces; ++i) bar_drain(full + 8 * i, (item - i + kPlaces - 1) / kPlaces, &dead);
        __syncwarp();
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    __syncwarp();
    if (wid == kWeighWarps)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * Z::kRows));
    if (tid == 0 && dead) kvq_error(v, kErrWaitLimit);
}

template <int D>
cudaError_t launch(WideArgs& p, bool bf, int sms, cudaStream_t stream) {
    using Z = Wide<D>;
    static_assert(Z::kBytes + 2560 <= 227 * 1024, "shared memory");  // and what the kernel has beside it
    const int64_t units = (int64_t)p.w.v.num_seqs * p.w.v.kv_heads;
    // one thread block for each SM where sequences and heads are fewer
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kMostSplits, sms / units));
    if (units * p.splits > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_after(bf ? kv_weigh_wide_kernel<D, true> : kv_weigh_wide_kernel<D, false>, units * p.splits, kThreads, Z::kBytes, stream, p);
}

}  // namespace

cudaError_t launch_kv_weigh_wide(const WeighArgs& a, int32_t head_dim, bool bf, int sms, cudaStream_t stream) {
    WideArgs p{};
    p.w = a, p.tries = prompt_wait_tries();
    if (cudaError_t e = kv_boxes(a.v, head_dim, bf, &p.boxes)) return e;
    return head_dim == 64 ? launch<64>(p, bf, sms, stream) : head_dim == 128 ? launch<128>(p, bf, sms, stream) : launch<256>(p, bf, sms, stream);
}

}  // namespace remp
