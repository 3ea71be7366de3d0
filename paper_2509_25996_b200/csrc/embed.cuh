// Rows gathered and scattered by token id, shared by the embedding, its gradient and the linear cross entropy.
#pragma once

#include "cast_internal.h"

namespace cast {

// Scratch of sort_tokens + scatter_rows over up to `tokens` tokens of width `dim`.
uint64_t scatter_scratch_bytes(int64_t tokens, int64_t dim);

// Order of the tokens by (id, position); ids outside [0, vocab) come last, as 0x7FFFFFFF.  Both arrays lie in `scratch`.
int sort_tokens(const int32_t* ids, int64_t tokens, int64_t vocab, int64_t dim, void* scratch, const int32_t** sorted_ids,
                const int32_t** order, cudaStream_t stream);

// dest[v] = scale * sum_{t: id = v} coef[t] src[t] over the sorted tokens (coef NULL: 1).  accumulate: added to dest, whose
// rows without a token are left alone; otherwise those rows become zero.
int scatter_rows(const uint16_t* src, const float* coef, float scale, const int32_t* sorted_ids, const int32_t* order, uint16_t* dest,
                 int64_t tokens, int64_t vocab, int64_t dim, bool accumulate, void* scratch, cudaStream_t stream);

// Address ranges [a, a + na) and [b, b + nb) share a byte.
inline bool ranges_overlap(const void* a, uint64_t na, const void* b, uint64_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + nb && y < x + na;
}

inline uint64_t align256(uint64_t n) { return (n + 255u) & ~255ull; }

}  // namespace cast
