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
    uint32_t* arrivals;     // counters of partial rows
    float* partial;
    int64_t tokens;
    bool few;               // so few that they are left as they came
    bool first;             // few, and no kernel of the call has been launched yet
};

// What the first kernel of a sort writes: ranked runs, and zeros to the counters.
struct SortStart {
    int32_t* ids;
    int32_t* order;
    uint32_t* arrivals;
    int64_t arrival_count;
};
SortStart sort_start(void* scratch, int64_t tokens, int64_t dim);

// Sorts into `scratch`: runs of kRun keys (rank_keys, launched here, or with `ranked` already done by rank_blocks() CTAs of the
// call's first kernel), then merges of the runs.
int rank_blocks(int64_t tokens);
int sort_tokens(bool ranked, const int32_t* ids, int64_t tokens, int64_t vocab, int64_t dim, void* scratch, SortedTokens* sorted, cudaStream_t stream);

// dest[v] = scale * sum_{t: id = v} src[t].  accumulate: added to dest, whose rows without a token are left alone; otherwise those
// become zero.
int scatter_rows(const SortedTokens& sorted, const uint16_t* src, float scale, uint16_t* dest, int64_t vocab, int64_t dim, bool accumulate,
                 cudaStream_t stream);

// The same sums as fp32 rows of their own, for a product's epilogue to add before its rounding: rows[row_of[v]] = sum_{t: id = v}
// coef[t] src[t].  `row_of` has an entry for every v, negative where no token has the id: the caller fills it before, the entries
// of ids in use are set here.  `rows` holds compact_rows() rows.  dim % 8 == 0, all aligned to 16 bytes.
inline int64_t compact_rows(int64_t tokens, int64_t vocab) { return tokens < vocab ? tokens : vocab; }
int gather_rows(const SortedTokens& sorted, const uint16_t* src, const float* coef, float* rows, int32_t* row_of, int64_t vocab, int64_t dim,
                cudaStream_t stream);

// Address ranges [a, a + na) and [b, b + nb) share a byte.
inline bool ranges_overlap(const void* a, uint64_t na, const void* b, uint64_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + nb && y < x + na;
}

// ------------------------------------------------------------------------------------------------ runs of keys

constexpr uint32_t kNoId = 0x7FFFFFFFu;
constexpr int kRun = 1024;            // keys ranked by counting
constexpr int kRankKeys = 128;        // keys of a run that one CTA places ...
constexpr int kRankShare = 4;         // ... with this many threads each
constexpr int kRankThreads = kRankKeys * kRankShare;

// One of `blocks` CTAs' part of ranking runs of kRun keys: a key's place is the number of keys of its run that come before it.
__device__ __forceinline__ void rank_keys(const int32_t* __restrict__ ids, const SortStart& start, int64_t tokens, uint32_t vocab, unsigned block,
                                          unsigned blocks)
{
    for (int64_t i = (int64_t)block * kRankThreads + threadIdx.x; i < start.arrival_count; i += (int64_t)blocks * kRankThreads) start.arrivals[i] = 0u;
    __shared__ uint4 keys4[kRun / 4];
    uint32_t* keys = reinterpret_cast<uint32_t*>(keys4);
    const int64_t run0 = (int64_t)(block / (kRun / kRankKeys)) * kRun;
    const int len = (int)min((int64_t)kRun, tokens - run0);
    const int first = (int)(block % (kRun / kRankKeys)) * kRankKeys;
    if (first >= len) return;             // uniform over the CTA
    const int n4 = (len + 3) / 4;
    for (int i = threadIdx.x; i < 4 * n4; i += kRankThreads) {
        // past the end: larger than every key, so that it comes before none
        uint32_t k = 0xFFFFFFFFu;
        if (i < len) {
            k = (uint32_t)ids[run0 + i];
            if (k >= vocab) k = kNoId;
        }
        keys[i] = k;
    }
    __syncthreads();
    const int p = min(first + (int)threadIdx.x / kRankShare, len - 1), share = (int)threadIdx.x % kRankShare;
    const uint32_t k = keys[p];
    const int own = p >> 2;
    int place = 0;
#pragma unroll 4
    for (int v = share; v < n4; v += kRankShare) {
        const uint4 o = keys4[v];
        const uint32_t limit = k + (v < own ? 1u : 0u);      // equal keys before this one count, equal keys after it do not
        place += (o.x < limit) + (o.y < limit) + (o.z < limit) + (o.w < limit);
    }
    if (share == 0)
        for (int j = 4 * own; j < p; ++j) place += keys[j] == k;
#pragma unroll
    for (int d = 1; d < kRankShare; d *= 2) place += __shfl_xor_sync(0xFFFFFFFFu, place, d);
    if (share == 0 && first + (int)threadIdx.x / kRankShare < len) {
        start.ids[run0 + place] = (int32_t)k;
        start.order[run0 + place] = (int32_t)(run0 + p);
    }
}

inline uint64_t align256(uint64_t n) { return (n + 255u) & ~255ull; }

}  // namespace cast
