// Rows gathered and scattered by token id, shared by the embedding, its gradient and the linear cross entropy.
#pragma once

#include "cast_internal.h"

namespace cast {

// Scratch of sort_tokens + scatter_rows over up to `tokens` tokens of width `dim`.
uint64_t scatter_scratch_bytes(int64_t tokens, int64_t dim);

// The tokens of a call in the order (id, position); ids outside [0, vocab) last, as 0x7FFFFFFF.
struct SortedTokens {
    const int32_t* ids;
    const int32_t* order;
    void* scratch;          // partial rows
    int64_t tokens;
};

// Sorts into `scratch`.  zeros: an array [vocab][dim] that is filled with zeros meanwhile, or NULL.  `first`: the first kernel of the call (see chained.cuh).
int sort_tokens(bool first, const int32_t* ids, int64_t tokens, int64_t vocab, int64_t dim, void* scratch, uint16_t* zeros, SortedTokens* sorted,
                cudaStream_t stream);

// dest[v] = scale * sum_{t: id = v} coef[t] src[t] (coef NULL: 1) for the rows that have a token; accumulate: added to what
// is there.
int scatter_rows(const SortedTokens& sorted, const uint16_t* src, const float* coef, float scale, uint16_t* dest, int64_t dim, bool accumulate,
                 cudaStream_t stream);

// Address ranges [a, a + na) and [b, b + nb) share a byte.
inline bool ranges_overlap(const void* a, uint64_t na, const void* b, uint64_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + nb && y < x + na;
}

inline uint64_t align256(uint64_t n) { return (n + 255u) & ~255ull; }

}  // namespace cast
