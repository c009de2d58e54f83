// Which rows and keys of a batch are a sequence's: whole-number arithmetic that no content of the caller's arrays and no window
// takes out of 32 bits (a compiler is free to turn a signed overflow into any index). No CUDA in it: it is tested on the host.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define REMP_HD __host__ __device__ __forceinline__
#else
#define REMP_HD static inline
#endif

namespace remp {

// Rows, sequences and tokens of a table's row stay below this, so that they can be rounded up to whole tiles and thread blocks.
constexpr int32_t kKvqMost = 0x7fff0000;

struct KvqSpan {
    int32_t q0, queries;  // first row of the call's tensors, rows
    int32_t len;          // cached tokens that the table's row can hold
    int32_t first_pos;    // position of the first row; negative where a sequence has more rows than tokens
};

// start, end: query_start[s], query_start[s + 1]; length: seq_lens[s]; room: tokens that a row of the table holds.
REMP_HD KvqSpan kvq_span(int32_t start, int32_t end, int32_t length, int32_t num_tokens, int32_t room) {
    const int32_t qs = start < 0 ? 0 : start > num_tokens ? num_tokens : start;
    const int32_t qe = end < qs ? qs : end > num_tokens ? num_tokens : end;
    const int32_t tokens = length < 0 ? 0 : length;
    return KvqSpan{qs, qe - qs, tokens > room ? room : tokens, tokens - (qe - qs)};
}

// The length does not fit the row, or a row stands before position 0.
REMP_HD bool kvq_span_bad(const KvqSpan& s, int32_t length) { return s.len != length || (s.queries > 0 && s.first_pos < 0); }

// The first key that a row at position `pos` sees (window 0: the first of all).
REMP_HD int32_t kvq_first_key(int32_t pos, int32_t window) { return window > 0 && pos >= window ? pos - window + 1 : 0; }

}  // namespace remp
