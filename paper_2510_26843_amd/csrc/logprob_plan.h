// How the log probabilities' rows are shared out (logprobs.hip), and the scratch of
// their parts.  Host code.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace cas {

// A part's record: m, s, u, and its K best: values, then ids.
static inline int lp_words(int K) { return 4 + 2 * K; }

// A row is walked by one workgroup of 1024 threads, or by workgroups of 256 in
// parts that k_logprob_join joins.  Measured, fp32 rows, in us:
// - One of 1024 where that walks a row in few chunks and the rows are about as many
//   as the CUs: 256 rows of 128256 logits, K = 20, 35 (in parts 45), 128 rows of
//   32000, K = 5, 11 (12 to 15).  A second round of them costs as much again (320
//   rows of 32000 22, in parts 19), and few rows leave CUs idle (48 of 128256,
//   K = 8, 21, in parts 13; but of 32000, one chunk, 64 rows 11 either way).
// - Parts of chunks of 8192 logits (32 a thread), or of 2048 (8 a thread: twice the
//   waves on a CU) where those would leave the chip empty (1 row of 128256, K = 5,
//   9.3 for 10.5), or mostly hold nothing (5000 rows of 1024 21 for 35), and for
//   many short rows (1501 of 32000 38 for 42; of 128256 128 for 110).
// - At most 64 parts: a lane of the join each (2 rows of 1000000 14.5, with 489 parts 18.6).
static constexpr int LP_PARTS = 64;
static constexpr int LP_SPAN = 32;  // most chunks of a part (at most 32: bits of a word)
struct LpPlan {
    int each, threads, parts, span;
};
static inline LpPlan lp_plan(int n, int V) {
    LpPlan p;
    const bool whole = n <= 256 && V > 16384 && V <= 131072 && (V <= 32768 || n > 64);
    const bool small = V <= 8192 || (n > 512 ? V <= 32768 : (int64_t)n * ((V + 8191) / 8192) < 512);
    p.threads = whole ? 1024 : 256;
    p.each = whole || !small ? 32 : 8;
    const int chunk = p.threads * p.each, chunks = (V + chunk - 1) / chunk;
    const int want = whole ? 1 : std::min({chunks, LP_PARTS, std::max(1, 2048 / n)});
    p.span = std::min((chunks + want - 1) / want, LP_SPAN);
    p.parts = (chunks + p.span - 1) / p.span;
    return p;
}
// The records of any call of up to n rows: those of 2048 parts, unless the rows'
// parts of LP_SPAN chunks are more.
static inline size_t lp_work_bytes(int n, int V, int K) {
    const int64_t most = std::min(LP_PARTS, (V + 2047) / 2048), least = (V + 8192 * LP_SPAN - 1) / (8192 * LP_SPAN);
    return (size_t)std::max(std::min(n * most, (int64_t)2048), n * least) * lp_words(K) * 4;
}

}  // namespace cas
