// Token embedding, out[t] = scale table[ids[t]], and its gradient, grad_table[v] = scale sum_{t: ids[t] = v} grad_out[t].
//
// Forward: a gather bounded by HBM (each output row written once, each table row in use read once).  One thread moves
// 16 bytes (8 columns); kUnroll of them per thread are in flight.  16384 tokens x 4096 columns whose frequencies fall like 1/rank
// (134 MB written, ~5500 different rows, 45 MB, read): 33 us, 5.4 TB/s; 8 tokens: 3 us, less than its launch from Python (10 us).
//
// Gradient: the tokens are put in the order (id, position) first, so that every table row sums its tokens in one fixed
// order, in fp32 registers, and is rounded and written once, without atomics: results do not change from run to run.
//   * sort: runs of 1024 are ranked by counting (a key's place = the keys of its run that come before it, an all-pairs
//     comparison from shared memory: 1024 comparisons per key, no passes and no histograms), then groups of 16 runs
//     are merged at once: a key's new place = its place in its own run + its bounds in the 15 others, found by binary
//     searches that advance together, so that their loads overlap.  16384 tokens take two launches, 262144 three.
//   * sums: a CTA takes kPiece sorted tokens and a block of columns, asks for all of its rows at once and stores the table rows
//     whose tokens all lie in its piece.  A table row whose tokens go on in the next piece leaves fp32 partial rows (the
//     part that enters a piece and the part that leaves it), which the warp that stores the last of them adds, in order.  Every
//     token row is read once, and a CTA's work does not depend on how often an id occurs.  (Letting a piece finish the row
//     that it leaves, where that ends in the next piece, saves partial rows but makes its loads a longer chain.)
//   * up to kFew tokens are not sorted: the first token of an id looks for the others among the ids (256 tokens x 768 added to a
//     table of 32000 rows: 12.4 us, sorted 14.3).
//   * rows without a token become zeros in further CTAs of the kernel that sums: each looks up which of its kZeroRows rows
//     the sorted ids hold, so nothing is written twice and the zeros share the bandwidth with the sums.  (Zeros beside the
//     ranking or the merge, whose latency they would hide, took 113 and 105 us where this took 97: writes alone are slower.)
// Bounded by HBM behind two short sorting kernels: 16384 tokens x 4096 into 32000 rows 91.5 us for 399 MB (4.3 TB/s; ranking and
// merging 13 us of it), 1000 tokens x 768 into 50257 rows 21 us for 79 MB.  More than kRun kWays = 16384 tokens take a second
// merge, whose searches go to L2: 16385 tokens 9 us longer; 32768 141 us (531 MB), 65536 233 (799 MB).  Adding to the table:
// 16384 97-99 us, 32768 181.
#include <cmath>
#include <type_traits>

#include "chained.cuh"
#include "embed.cuh"

namespace cast {
namespace {

constexpr int kWays = 16;           // runs merged at once
constexpr int kPiece = 16;          // sorted tokens per CTA

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// VEC = 8 columns (16 bytes) or 1 column per access.
template <int VEC> struct Cols;
template <> struct Cols<8> {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    using Raw = uint4;
    static __device__ __forceinline__ Raw load(const uint16_t* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void add(const Raw& x, float c) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = fmaf(c, bf16_lo(w[i]), v[2 * i]); v[2 * i + 1] = fmaf(c, bf16_hi(w[i]), v[2 * i + 1]); }
    }
    // a partial row that another SM may have written in this kernel: from L2
    __device__ __forceinline__ void add_partial(const float* p) {
        const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    __device__ __forceinline__ void add(const Cols& o) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += o.v[i];
    }
    __device__ __forceinline__ void store_partial(float* p) const {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    static __device__ __forceinline__ Raw load_own(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }      // memory this kernel writes
    // scale times the sums, added to `old` or not, rounded once
    __device__ __forceinline__ void store(uint16_t* p, float scale, bool add, const Raw& old) const {
        uint4* q = reinterpret_cast<uint4*>(p);
        const uint32_t o[4] = {add ? old.x : 0u, add ? old.y : 0u, add ? old.z : 0u, add ? old.w : 0u};
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack_bf16(fmaf(scale, v[2 * i], bf16_lo(o[i])), fmaf(scale, v[2 * i + 1], bf16_hi(o[i])));
        __stcs(q, make_uint4(r[0], r[1], r[2], r[3]));
    }
};
template <> struct Cols<1> {
    float v;
    __device__ __forceinline__ void zero() { v = 0.0f; }
    using Raw = uint16_t;
    static __device__ __forceinline__ Raw load(const uint16_t* p) { return __ldg(p); }
    __device__ __forceinline__ void add(Raw x, float c) { v = fmaf(c, bf16_lo(x), v); }
    __device__ __forceinline__ void add_partial(const float* p) { v += __ldcg(p); }
    __device__ __forceinline__ void add(const Cols& o) { v += o.v; }
    __device__ __forceinline__ void store_partial(float* p) const { *p = v; }
    static __device__ __forceinline__ Raw load_own(const uint16_t* p) { return *p; }
    __device__ __forceinline__ void store(uint16_t* p, float scale, bool add, Raw old) const {
        *p = (uint16_t)(pack_bf16(fmaf(scale, v, add ? bf16_lo(old) : 0.0f), 0.0f) & 0xFFFFu);
    }
};

// ------------------------------------------------------------------------------------------------ forward

constexpr int kEmbedThreads = 256;
constexpr int kUnroll = 4;

template <int VEC>
__global__ void __launch_bounds__(kEmbedThreads)
embed_kernel(const uint16_t* __restrict__ table, const int32_t* __restrict__ ids, uint16_t* __restrict__ out, int64_t n_units,
             uint32_t units_per_row, uint32_t vocab, float scale)
{
    using Raw = typename std::conditional<VEC == 8, uint4, uint16_t>::type;
    const int64_t first = (int64_t)blockIdx.x * (kEmbedThreads * kUnroll) + threadIdx.x;
    Raw x[kUnroll];
    bool have[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const int64_t u = first + i * kEmbedThreads;
        have[i] = false;
        if (u < n_units) {
            const int64_t token = u / units_per_row;
            const uint32_t c = (uint32_t)(u - token * units_per_row);
            const uint32_t id = (uint32_t)__ldg(ids + token);
            have[i] = id < vocab;
            if (have[i]) x[i] = __ldg(reinterpret_cast<const Raw*>(table) + (int64_t)id * units_per_row + c);
        }
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const int64_t u = first + i * kEmbedThreads;
        if (u >= n_units) continue;
        if constexpr (VEC == 8) {
            uint4 r = make_uint4(0u, 0u, 0u, 0u);
            if (have[i])
                r = make_uint4(pack_bf16(scale * bf16_lo(x[i].x), scale * bf16_hi(x[i].x)), pack_bf16(scale * bf16_lo(x[i].y), scale * bf16_hi(x[i].y)),
                               pack_bf16(scale * bf16_lo(x[i].z), scale * bf16_hi(x[i].z)), pack_bf16(scale * bf16_lo(x[i].w), scale * bf16_hi(x[i].w)));
            reinterpret_cast<uint4*>(out)[u] = r;
        } else {
            out[u] = have[i] ? (uint16_t)(pack_bf16(scale * bf16_lo(x[i]), 0.0f) & 0xFFFFu) : (uint16_t)0;
        }
    }
}

// ------------------------------------------------------------------------------------------------ order of the tokens

__global__ void __launch_bounds__(kRankThreads)
rank_runs_kernel(const int32_t* __restrict__ ids, const SortStart start, int64_t tokens, uint32_t vocab)
{
    chain_next();
    chain_wait();
    rank_keys(ids, start, tokens, vocab, blockIdx.x, gridDim.x);
}

constexpr int kMergeKeys = 128;                   // per CTA ...
constexpr int kMergeShare = 8;                    // ... searched for by this many threads each
constexpr int kMergeThreads = kMergeKeys * kMergeShare;

// Merges groups of kWays runs of `run` keys.  A thread's searches advance together and without branches: independent loads in
// each halving, from shared memory where a group fits (runs of kRun keys: 64 KB), from L2 where it does not.
template <bool SHARED>
__global__ void __launch_bounds__(kMergeThreads)
merge_runs_kernel(const int32_t* __restrict__ ids_in, const int32_t* __restrict__ order_in, int32_t* __restrict__ ids_out,
                  int32_t* __restrict__ order_out, int32_t tokens, int32_t run)
{
    extern __shared__ int32_t group_ids[];
    chain_next();
    chain_wait();
    const int share = (int)threadIdx.x % kMergeShare;
    const int64_t place = (int64_t)blockIdx.x * kMergeKeys + (int)threadIdx.x / kMergeShare;
    const int32_t i = (int32_t)min(place, (int64_t)tokens - 1), from = __ldg(order_in + i);
    const int64_t group = (int64_t)run * kWays;
    const int32_t group0 = (int32_t)((int64_t)blockIdx.x * kMergeKeys / group * group);      // of the CTA: its keys are of one run
    const int32_t left = tokens - group0;            // keys of the group, and of the groups after it
    const int32_t* keys = ids_in + group0;
    if constexpr (SHARED) {
        const int32_t n4 = (min(left, kRun * kWays) + 3) / 4;      // the arrays are padded to whole vectors
#pragma unroll 8
        for (int32_t v = threadIdx.x; v < n4; v += kMergeThreads)
            reinterpret_cast<int4*>(group_ids)[v] = __ldg(reinterpret_cast<const int4*>(keys) + v);
        __syncthreads();
        keys = group_ids;
    }
    const int own = (i - group0) / run;
    const uint32_t k = (uint32_t)keys[i - group0];
    constexpr int kEach = kWays / kMergeShare;
    int32_t pos[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) pos[j] = 0;
    for (int32_t half = run; half; half >>= 1) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = j * kMergeShare + share;
            const int64_t before = (int64_t)r * run;                 // keys of the group ahead of run r
            const int32_t at = pos[j] + half;
            const bool there = at <= run && before + at <= left;
            const uint32_t limit = r == own ? 0u : k + (r < own ? 1u : 0u);
            const uint32_t other = (uint32_t)keys[there ? (int32_t)before + at - 1 : 0];
            pos[j] = there && other < limit ? at : pos[j];
        }
    }
    int32_t ahead = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) ahead += pos[j];
#pragma unroll
    for (int d = 1; d < kMergeShare; d *= 2) ahead += __shfl_xor_sync(0xFFFFFFFFu, ahead, d);
    if (share == 0 && place < tokens) {
        const int32_t to = group0 + (i - group0 - own * run) + ahead;
        ids_out[to] = (int32_t)k;
        order_out[to] = from;
    }
}

// ------------------------------------------------------------------------------------------------ sums

constexpr int kScatterThreads = 256;

// What becomes of a sum: a bf16 row of the table, written or added to, or an fp32 row of its own (gather_rows).
enum class Into { kTable, kAdded, kRows };

struct ScatterArgs {
    const uint16_t* src;
    const float* coef;            // per token (kRows)
    const int32_t* ids;           // sorted
    const int32_t* order;
    float* partial;               // [pieces][2][dim]: what enters a piece, what leaves it
    uint32_t* arrivals;           // [2 pieces + groups][warp columns], zero
    uint16_t* dest;               // kTable, kAdded
    float* rows;                  // kRows
    int32_t* row_of;
    int64_t dim, vocab;
    int32_t tokens, pieces;
    unsigned own, columns;        // CTAs that sum: own / columns for the tokens x columns; the ones after them write zeros
    float scale;
    int lanes;                    // threads per row: 32 .. 256, a power of two
};

// A finished sum.  `place`: a sorted position (of few tokens, a token) that is this id's alone, by which its row of kRows goes where
// there are fewer tokens than ids.
template <int VEC, Into INTO>
__device__ __forceinline__ void store_sum(const ScatterArgs& a, const Cols<VEC>& acc, int32_t id, int32_t place, int32_t col, const typename Cols<VEC>::Raw& old)
{
    if constexpr (INTO == Into::kRows) {
        const int32_t row = a.tokens > a.vocab ? id : place;
        acc.store_partial(a.rows + (int64_t)row * a.dim + col);
        if (col == 0) a.row_of[id] = row;
    } else {
        acc.store(a.dest + (int64_t)id * a.dim + col, a.scale, INTO == Into::kAdded, old);
    }
}

// Column of this thread: a.lanes threads per row, the rest of a long row in the CTAs beside it.
template <int VEC>
__device__ __forceinline__ int32_t column_of(const ScatterArgs& a)
{
    return ((int32_t)(blockIdx.x % a.columns) * a.lanes + (int)threadIdx.x % a.lanes) * VEC;
}

// First sorted position with an id of at least `id`, found by the 32 lanes of a warp together (32 ways per step).
__device__ __forceinline__ int32_t warp_lower_bound(const int32_t* ids, int32_t n, int64_t id)
{
    const int lane = (int)threadIdx.x & 31;
    int32_t lo = 0, hi = n;                       // the answer is in [lo, hi]
    while (lo < hi) {
        const int32_t step = (hi - lo + 31) / 32;
        const int64_t at = (int64_t)lo + (int64_t)(lane + 1) * step - 1;          // last position of this lane's part
        const bool less = at < hi && (int64_t)__ldg(ids + at) < id;
        const int parts = __popc(__ballot_sync(0xFFFFFFFFu, less));
        lo += parts * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

constexpr int kZeroRows = 32;

// Writes the rows without a token among rows [row0, row0 + kZeroRows); `held`: bit i for row0 + i.
template <int VEC>
__device__ __forceinline__ void zero_rows(const ScatterArgs& a, int64_t row0, uint32_t held)
{
    using Raw = typename Cols<VEC>::Raw;
    const uint32_t per = (uint32_t)(a.dim / VEC);
    if (per >= (unsigned)kScatterThreads) {
        for (int r = 0; r < kZeroRows && row0 + r < a.vocab; ++r) {
            if (held >> r & 1u) continue;
            Raw* to = reinterpret_cast<Raw*>(a.dest + (row0 + r) * a.dim);
            for (uint32_t i = threadIdx.x; i < per; i += kScatterThreads) __stcs(to + i, Raw{});
        }
    } else {
        Raw* to = reinterpret_cast<Raw*>(a.dest + row0 * a.dim);
        const uint32_t rows = (uint32_t)min((int64_t)kZeroRows, a.vocab - row0);
        for (uint32_t i = threadIdx.x; i < rows * per; i += kScatterThreads)
            if (!(held >> (i / per) & 1u)) __stcs(to + i, Raw{});
    }
}

// A CTA past the ones that sum: finds out which rows of its block the sorted ids hold, and writes the others.
template <int VEC>
__device__ __forceinline__ void zero_block(const ScatterArgs& a)
{
    __shared__ int32_t range[2];
    __shared__ uint32_t held;
    const int64_t row0 = (int64_t)(blockIdx.x - a.own) * kZeroRows;
    const int warp = (int)threadIdx.x >> 5;
    if (threadIdx.x == 0) held = 0;
    if (warp < 2) {
        const int32_t b = warp_lower_bound(a.ids, a.tokens, row0 + (warp ? kZeroRows : 0));
        if ((threadIdx.x & 31) == 0) range[warp] = b;
    }
    __syncthreads();
    for (int32_t p = range[0] + (int)threadIdx.x; p < range[1]; p += kScatterThreads) {
        const int64_t id = __ldg(a.ids + p);
        if (id < a.vocab) atomicOr(&held, 1u << (int)(id - row0));       // a block that ends past the vocabulary also sees the ids that are none
    }
    __syncthreads();
    zero_rows<VEC>(a, row0, held);
}

// ------------------------------------------------------------------------------------------------ rows of several pieces

// A table row whose tokens lie in several pieces has a partial row in each: what left the first, what entered the others.  Each warp
// that has stored one counts itself in, and the last one adds them all, in the order of the pieces; nobody waits.  Pieces are
// counted in groups of kGroup (aligned, so that the order of the additions depends on the sorted ids alone); a row of several
// groups, a frequent token's, is joined from the groups' sums in the same way.
constexpr int kGroup = 16;

// The id that crosses the start of a piece (the token before it and its first one have it), -1 where none does.
__device__ __forceinline__ int32_t crossing(const ScatterArgs& a, int64_t piece)
{
    const int64_t p = piece * kPiece;
    if (p <= 0 || p >= a.tokens) return -1;
    const int32_t before = __ldg(a.ids + p - 1), first = __ldg(a.ids + p);
    return before == first ? first : -1;
}

// The warp has stored its part; whether all `parts` of this counter have been.
__device__ __forceinline__ bool arrive_last(uint32_t* counter, int32_t parts)
{
    __threadfence();
    __syncwarp();
    uint32_t before = 0;
    if ((threadIdx.x & 31) == 0) before = atomicAdd(counter, 1u);
    before = __shfl_sync(0xFFFFFFFFu, before, 0);
    if (before + 1 != (uint32_t)parts) return false;
    __threadfence();
    return true;
}

// Rows p, p + stride, ... of `count`, four at a time, the last ones too.
template <int VEC>
__device__ __forceinline__ void add_partials(Cols<VEC>& acc, const float* p, int64_t stride, int32_t count)
{
    for (int32_t i = 0; i < count; i += 4) {
        Cols<VEC> row[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            row[j].zero();
            if (i + j < count) row[j].add_partial(p + (int64_t)(i + j) * stride);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) acc.add(row[j]);
    }
}

// `crossed`: of the row with this id, bit j for the start of piece kGroup group + j, j <= kGroup.  A whole warp; `in`: this lane has columns.
template <int VEC, Into INTO>
__device__ __forceinline__ void join_row(const ScatterArgs& a, int32_t id, uint32_t crossed, int32_t group, int32_t col, int32_t warp_col, int32_t warp_cols, bool in)
{
    const int lane = (int)threadIdx.x & 31;
    const int32_t piece0 = group * kGroup, low = __ffs((int)crossed) - 1;
    const bool begins = low > 0, goes_on = crossed >> kGroup & 1u;              // the row's first token is in this group; its last one is not
    const int32_t entered = __popc(crossed & ((1u << kGroup) - 1u));            // pieces of the group that it enters
    const int64_t row0 = begins ? 2 * (int64_t)(piece0 + low - 1) + 1 : 2 * (int64_t)piece0;      // its first partial row in the group
    if (!arrive_last(a.arrivals + row0 * warp_cols + warp_col, entered + (begins ? 1 : 0))) return;
    int32_t place = (piece0 + low) * kPiece;                                     // where it enters a piece for the first time
    Cols<VEC> acc;
    acc.zero();
    if (in) {
        if (begins) acc.add_partial(a.partial + row0 * a.dim + col);
        add_partials<VEC>(acc, a.partial + 2 * (int64_t)(piece0 + low) * a.dim + col, 2 * a.dim, entered);
    }
    if (!begins || goes_on) {
        if (in) acc.store_partial(a.partial + row0 * a.dim + col);             // the group's sum, where its first row was
        int32_t head = group, tail = group;                                     // the groups with the row's first and last token
        for (bool more = !begins; more;) {
            const int32_t g = head - 1 - lane;                                  // does it enter this group, too?
            const uint32_t no = ~__ballot_sync(0xFFFFFFFFu, crossing(a, (int64_t)g * kGroup) == id);
            head -= no ? __ffs((int)no) : 32;
            more = !no;
        }
        for (bool more = goes_on; more;) {
            const int32_t g = tail + 2 + lane;
            const uint32_t no = ~__ballot_sync(0xFFFFFFFFu, crossing(a, (int64_t)g * kGroup) == id);
            tail += no ? __ffs((int)no) : 32;
            more = !no;
        }
        // only one row goes on from a group to the next
        if (!arrive_last(a.arrivals + (2 * (int64_t)a.pieces + head) * warp_cols + warp_col, tail - head + 1)) return;
        const uint32_t starts = __ballot_sync(0xFFFFFFFFu, lane <= kGroup && crossing(a, (int64_t)head * kGroup + lane) == id);
        place = (head * kGroup + __ffs((int)starts) - 1) * kPiece;
        acc.zero();
        if (in) {
            acc.add_partial(a.partial + (2 * (int64_t)(head * kGroup + __ffs((int)starts) - 2) + 1) * a.dim + col);
            add_partials<VEC>(acc, a.partial + 2 * (int64_t)(head + 1) * kGroup * a.dim + col, 2 * kGroup * a.dim, tail - head);
        }
    }
    if (!in) return;
    typename Cols<VEC>::Raw old = {};
    if constexpr (INTO == Into::kAdded) old = Cols<VEC>::load_own(a.dest + (int64_t)id * a.dim + col);
    store_sum<VEC, INTO>(a, acc, id, place, col, old);
}

// One piece of kPiece sorted tokens per group of a.lanes threads.  kAdded: what is there is asked for together with the token
// rows, which would otherwise be one dependent load after the other.
template <int VEC, Into INTO>
__global__ void __launch_bounds__(kScatterThreads, INTO == Into::kTable ? 3 : 2)
piece_sums_kernel(const __grid_constant__ ScatterArgs a)
{
    constexpr int kBatch = 8;             // token rows asked for at a time
    constexpr bool COEF = INTO == Into::kRows, ACC = INTO == Into::kAdded;
    chain_next();
    chain_wait();
    if constexpr (INTO == Into::kTable) {
        if (blockIdx.x >= a.own) {
            zero_block<VEC>(a);
            return;
        }
    }
    const int32_t piece = (int32_t)(blockIdx.x / a.columns) * (kScatterThreads / a.lanes) + (int)threadIdx.x / a.lanes;
    if (piece >= a.pieces) return;
    const int32_t col = column_of<VEC>(a);
    const bool in = col < a.dim;
    const int32_t p0 = piece * kPiece, n = min(kPiece, a.tokens - p0);
    // the ids of the piece, the one before it and the one after it; 0xFFFFFFFF where there is none
    uint32_t id[kPiece + 2];
    int32_t t[kPiece];
#pragma unroll
    for (int i = 0; i < kPiece + 2; ++i) {
        const int32_t p = p0 + i - 1;
        id[i] = p >= 0 && p < a.tokens ? (uint32_t)__ldg(a.ids + p) : 0xFFFFFFFFu;
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i) t[i] = in && i < n && id[i + 1] != kNoId ? __ldg(a.order + p0 + i) : -1;
    const int lane = (int)threadIdx.x & 31;
    const int32_t group = piece / kGroup, crosses = lane <= kGroup ? crossing(a, (int64_t)group * kGroup + lane) : -1;
    const uint16_t* src = a.src + col;
    float* partial = a.partial + (int64_t)piece * 2 * a.dim + col;
    bool entered = id[0] == id[1];        // the current row's tokens began in an earlier piece
    Cols<VEC> acc;
    acc.zero();
#pragma unroll
    for (int b = 0; b < kPiece; b += kBatch) {
        typename Cols<VEC>::Raw x[kBatch], old[ACC ? kBatch : 1];
        float c[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            c[i] = 1.0f;
            if (t[b + i] >= 0) {
                x[i] = Cols<VEC>::load(src + (int64_t)t[b + i] * a.dim);
                if constexpr (COEF) c[i] = __ldg(a.coef + t[b + i]);
                if constexpr (ACC)
                    if (id[b + i + 2] != id[b + i + 1]) old[i] = Cols<VEC>::load_own(a.dest + (int64_t)id[b + i + 1] * a.dim + col);
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (t[b + i] < 0) continue;
            acc.add(x[i], c[i]);
            const uint32_t own = id[b + i + 1];
            if (id[b + i + 2] != own) {                    // its last token
                if (entered) acc.store_partial(partial);
                else store_sum<VEC, INTO>(a, acc, (int32_t)own, p0 + b + i, col, old[ACC ? i : 0]);
                entered = false;
                acc.zero();
            } else if (b + i == kPiece - 1) {              // goes on in the next piece
                acc.store_partial(entered ? partial : partial + a.dim);
            }
        }
    }
    const bool enters = id[0] == id[1] && id[1] != kNoId, leaves = id[kPiece] == id[kPiece + 1] && id[kPiece] < kNoId;
    const int32_t warp_col = col / (32 * VEC), warp_cols = (int32_t)a.columns * (a.lanes / 32);
    if (enters) join_row<VEC, INTO>(a, (int32_t)id[1], __ballot_sync(0xFFFFFFFFu, crosses == (int32_t)id[1]), group, col, warp_col, warp_cols, in);
    if (leaves && !(enters && id[kPiece] == id[1]))
        join_row<VEC, INTO>(a, (int32_t)id[kPiece], __ballot_sync(0xFFFFFFFFu, crosses == (int32_t)id[kPiece]), group, col, warp_col, warp_cols, in);
}

// Few tokens need no order: the threads that hold an id's first token list the others by warp votes over all ids.
constexpr int kFew = 256;

template <int VEC, Into INTO>
__global__ void __launch_bounds__(kScatterThreads)
few_tokens_kernel(const __grid_constant__ ScatterArgs a, uint32_t vocab)      // a.ids: as the caller gave them
{
    constexpr int kWarps = kScatterThreads / 32;
    __shared__ uint32_t ids[kFew];
    __shared__ uint8_t same[kWarps][kFew];
    __shared__ uint32_t held;
    chain_next();
    if (threadIdx.x == 0) held = 0;
    ids[threadIdx.x] = (int)threadIdx.x < a.tokens ? (uint32_t)__ldg(a.ids + threadIdx.x) : 0xFFFFFFFFu;
    __syncthreads();
    if (blockIdx.x >= a.own) {           // a block of rows: zeros where no token is (kTable)
        chain_wait();
        const int64_t row0 = (int64_t)(blockIdx.x - a.own) * kZeroRows;
        const int64_t id = (int64_t)ids[threadIdx.x] - row0;
        if (ids[threadIdx.x] < vocab && id >= 0 && id < kZeroRows) atomicOr(&held, 1u << (int)id);
        __syncthreads();
        zero_rows<VEC>(a, row0, held);
        return;
    }
    const int32_t t = (int32_t)(blockIdx.x / a.columns) * (kScatterThreads / a.lanes) + (int)threadIdx.x / a.lanes;      // one token per warp
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const uint32_t id = t < a.tokens ? ids[t] : 0xFFFFFFFFu;
    // Every thread waits for the predecessor, those without a row to add too: what follows the call waits for this grid alone, and a
    // grid of which no thread had waited (no token has an id) could end before its predecessor.
    if (id >= vocab) {
        chain_wait();
        return;
    }
    int count = 0;
#pragma unroll
    for (int k = 0; k < kFew / 32; ++k) {
        const bool mine = ids[32 * k + lane] == id;
        const uint32_t m = __ballot_sync(0xFFFFFFFFu, mine);
        if (mine) same[warp][count + __popc(m & ((1u << lane) - 1u))] = (uint8_t)(32 * k + lane);
        count += __popc(m);
    }
    __syncwarp();
    const bool first = same[warp][0] == t;
    const int32_t col = column_of<VEC>(a);
    chain_wait();
    if (!first || col >= a.dim) return;
    typename Cols<VEC>::Raw old = {};
    if constexpr (INTO == Into::kAdded) old = Cols<VEC>::load_own(a.dest + (int64_t)id * a.dim + col);
    Cols<VEC> acc;
    acc.zero();
    for (int32_t i0 = 0; i0 < count; i0 += 4) {
        typename Cols<VEC>::Raw x[4];
        float c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = 1.0f;
            if (i0 + i < count) {
                const int32_t token = same[warp][i0 + i];
                x[i] = Cols<VEC>::load(a.src + (int64_t)token * a.dim + col);
                if constexpr (INTO == Into::kRows) c[i] = __ldg(a.coef + token);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i0 + i < count) acc.add(x[i], c[i]);
    }
    store_sum<VEC, INTO>(a, acc, (int32_t)id, t, col, old);
}

template <int VEC, Into INTO>
int launch_scatter(ScatterArgs a, const SortedTokens& sorted, cudaStream_t stream)
{
    const int64_t units = (a.dim + VEC - 1) / VEC;
    a.lanes = 32;
    while (a.lanes < kScatterThreads && a.lanes < units) a.lanes *= 2;
    const int64_t groups = kScatterThreads / a.lanes, items = sorted.few ? a.tokens : a.pieces;
    a.columns = (unsigned)((units + a.lanes - 1) / a.lanes);
    a.own = (unsigned)((items + groups - 1) / groups) * a.columns;
    const unsigned zeros = INTO == Into::kTable ? (unsigned)((a.vocab + kZeroRows - 1) / kZeroRows) : 0u;
    const dim3 grid(a.own + zeros);
    if (sorted.few) return launch_chained(sorted.first, few_tokens_kernel<VEC, INTO>, grid, kScatterThreads, 0, stream, 1, a, (uint32_t)a.vocab);
    return launch_chained(false, piece_sums_kernel<VEC, INTO>, grid, kScatterThreads, 0, stream, 1, a);
}

ScatterArgs scatter_args(const SortedTokens& sorted, const uint16_t* src, int64_t vocab, int64_t dim)
{
    ScatterArgs a = {};
    a.src = src;
    a.ids = sorted.ids;
    a.order = sorted.order;
    a.partial = sorted.partial;
    a.arrivals = sorted.arrivals;
    a.tokens = (int32_t)sorted.tokens;
    a.pieces = (int32_t)((sorted.tokens + kPiece - 1) / kPiece);
    a.dim = dim;
    a.vocab = vocab;
    a.scale = 1.0f;
    return a;
}

int64_t sort_array_bytes(int64_t tokens) { return (int64_t)align256(4ull * (uint64_t)tokens); }

int64_t pieces_of(int64_t tokens) { return (tokens + kPiece - 1) / kPiece; }

// Counters of join_row: two per piece and one per group, for each warp of columns (at most: one column per lane).
int64_t arrival_count(int64_t tokens, int64_t dim)
{
    const int64_t pieces = pieces_of(tokens);
    return (2 * pieces + (pieces + kGroup - 1) / kGroup) * ((dim + kScatterThreads - 1) / kScatterThreads * (kScatterThreads / 32));
}

}  // namespace

uint64_t scatter_scratch_bytes(int64_t tokens, int64_t dim)
{
    // two copies of (sorted ids, order), the counters, the partial rows
    return 4ull * (uint64_t)sort_array_bytes(tokens) + align256(4ull * (uint64_t)arrival_count(tokens, dim)) +
           align256(8ull * (uint64_t)pieces_of(tokens) * (uint64_t)dim);
}

SortStart sort_start(void* scratch, int64_t tokens, int64_t dim)
{
    const int64_t step = sort_array_bytes(tokens);
    uint8_t* b = static_cast<uint8_t*>(scratch);
    return {reinterpret_cast<int32_t*>(b), reinterpret_cast<int32_t*>(b + step), reinterpret_cast<uint32_t*>(b + 4 * step), arrival_count(tokens, dim)};
}

int rank_blocks(int64_t tokens) { return tokens <= kFew ? 0 : (int)((tokens + kRun - 1) / kRun * (kRun / kRankKeys)); }

int sort_tokens(bool ranked, const int32_t* ids, int64_t tokens, int64_t vocab, int64_t dim, void* scratch, SortedTokens* sorted, cudaStream_t stream)
{
    *sorted = {};
    sorted->tokens = tokens;
    if (tokens <= kFew) {
        sorted->few = true;
        sorted->ids = ids;
        sorted->first = !ranked;
        return CAST_OK;
    }
    const SortStart start = sort_start(scratch, tokens, dim);
    const int64_t step = sort_array_bytes(tokens) / 4;
    int32_t *const id_buf[2] = {start.ids, start.ids + 2 * step}, *const or_buf[2] = {start.order, start.order + 2 * step};
    int rc;
    if (!ranked && (rc = launch_chained(true, rank_runs_kernel, dim3((unsigned)rank_blocks(tokens)), kRankThreads, 0, stream, 1, ids, start, tokens,
                                        (uint32_t)vocab)) != CAST_OK)
        return rc;
    int cur = 0;
    for (int64_t run = kRun; run < tokens; run *= kWays, cur ^= 1) {
        const dim3 grid((unsigned)((tokens + kMergeKeys - 1) / kMergeKeys));
        if (run == kRun) {
            constexpr size_t smem = sizeof(int32_t) * kRun * kWays;
            CAST_CUDA_TRY(cudaFuncSetAttribute(merge_runs_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
            rc = launch_chained(false, merge_runs_kernel<true>, grid, kMergeThreads, smem, stream, 1, id_buf[cur], or_buf[cur], id_buf[cur ^ 1],
                                or_buf[cur ^ 1], (int32_t)tokens, (int32_t)run);
        } else {
            rc = launch_chained(false, merge_runs_kernel<false>, grid, kMergeThreads, 0, stream, 1, id_buf[cur], or_buf[cur], id_buf[cur ^ 1],
                                or_buf[cur ^ 1], (int32_t)tokens, (int32_t)run);
        }
        if (rc != CAST_OK) return rc;
    }
    sorted->ids = id_buf[cur];
    sorted->order = or_buf[cur];
    sorted->arrivals = start.arrivals;
    sorted->partial = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(start.arrivals) + align256(4ull * (uint64_t)start.arrival_count));
    return CAST_OK;
}

int scatter_rows(const SortedTokens& sorted, const uint16_t* src, float scale, uint16_t* dest, int64_t vocab, int64_t dim, bool accumulate,
                 cudaStream_t stream)
{
    ScatterArgs a = scatter_args(sorted, src, vocab, dim);
    a.dest = dest;
    a.scale = scale;
    const bool vec = dim % 8 == 0 && !((uintptr_t)src & 15u) && !((uintptr_t)dest & 15u);
    if (vec) return accumulate ? launch_scatter<8, Into::kAdded>(a, sorted, stream) : launch_scatter<8, Into::kTable>(a, sorted, stream);
    return accumulate ? launch_scatter<1, Into::kAdded>(a, sorted, stream) : launch_scatter<1, Into::kTable>(a, sorted, stream);
}

int gather_rows(const SortedTokens& sorted, const uint16_t* src, const float* coef, float* rows, int32_t* row_of, int64_t vocab, int64_t dim,
                cudaStream_t stream)
{
    ScatterArgs a = scatter_args(sorted, src, vocab, dim);
    a.coef = coef;
    a.rows = rows;
    a.row_of = row_of;
    return launch_scatter<8, Into::kRows>(a, sorted, stream);
}

}  // namespace cast

using namespace cast;

namespace {

constexpr int64_t kMostColumns = 1 << 20;      // blocks of 32 accesses of one column each: fewer than 2^16

int check_rows(const void* a, const void* ids, const void* b, int64_t tokens, int64_t vocab, int64_t dim, float scale)
{
    if (!a || !ids || !b) return CAST_ERR_NULL;
    if (tokens < 1 || vocab < 1 || dim < 1 || tokens > 0x3FFFFFFF || vocab > 0x7FFFFFFE || dim > kMostColumns) return CAST_ERR_SHAPE;
    if (vocab > ((int64_t)1 << 40) / dim || tokens > ((int64_t)1 << 40) / dim) return CAST_ERR_SHAPE;
    if (!std::isfinite(scale)) return CAST_ERR_HYPER;
    if (((uintptr_t)a & 1u) || ((uintptr_t)b & 1u) || ((uintptr_t)ids & 3u)) return CAST_ERR_ALIGN;
    return CAST_OK;
}

}  // namespace

extern "C" int cast_embed(const cast_bf16* table, const int32_t* ids, cast_bf16* out, int64_t tokens, int64_t vocab, int64_t dim,
                          float scale, cast_stream_t stream)
{
    int rc;
    if ((rc = check_rows(table, ids, out, tokens, vocab, dim, scale)) != CAST_OK) return rc;
    const uint64_t out_bytes = 2ull * (uint64_t)tokens * (uint64_t)dim;
    if (ranges_overlap(out, out_bytes, table, 2ull * (uint64_t)vocab * (uint64_t)dim) || ranges_overlap(out, out_bytes, ids, 4ull * (uint64_t)tokens))
        return CAST_ERR_ALIAS;
    const void* ptrs[3] = {table, ids, out};
    if ((rc = check_device_memory(ptrs, 3)) != CAST_OK) return rc;
    const bool vec = dim % 8 == 0 && !((uintptr_t)table & 15u) && !((uintptr_t)out & 15u);
    const int64_t per_row = vec ? dim / 8 : dim, units = tokens * per_row;
    const int64_t grid = (units + kEmbedThreads * kUnroll - 1) / (kEmbedThreads * kUnroll);
    if (grid > 0x7FFFFFFF) return CAST_ERR_SHAPE;
    cudaStream_t s = (cudaStream_t)stream;
    if (vec) embed_kernel<8><<<(unsigned)grid, kEmbedThreads, 0, s>>>(table, ids, out, units, (uint32_t)per_row, (uint32_t)vocab, scale);
    else embed_kernel<1><<<(unsigned)grid, kEmbedThreads, 0, s>>>(table, ids, out, units, (uint32_t)per_row, (uint32_t)vocab, scale);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    return CAST_OK;
}

extern "C" int cast_embed_grad_workspace(int64_t tokens, int64_t dim, uint64_t* bytes)
{
    if (!bytes) return CAST_ERR_NULL;
    if (tokens < 1 || dim < 1 || tokens > 0x3FFFFFFF || dim > kMostColumns || tokens > ((int64_t)1 << 40) / dim) return CAST_ERR_SHAPE;
    *bytes = scatter_scratch_bytes(tokens, dim);
    return CAST_OK;
}

extern "C" int cast_embed_grad(const cast_bf16* grad_out, const int32_t* ids, cast_bf16* grad_table, int64_t tokens, int64_t vocab,
                               int64_t dim, float scale, int accumulate, void* workspace, uint64_t workspace_bytes, cast_stream_t stream)
{
    int rc;
    if ((rc = check_rows(grad_out, ids, grad_table, tokens, vocab, dim, scale)) != CAST_OK) return rc;
    if (!workspace) return CAST_ERR_NULL;
    if ((uintptr_t)workspace & 15u) return CAST_ERR_ALIGN;
    const uint64_t need = scatter_scratch_bytes(tokens, dim);
    if (workspace_bytes < need) return CAST_ERR_PLAN;
    const uint64_t in_bytes = 2ull * (uint64_t)tokens * (uint64_t)dim, table_bytes = 2ull * (uint64_t)vocab * (uint64_t)dim;
    if (ranges_overlap(grad_table, table_bytes, grad_out, in_bytes) || ranges_overlap(grad_table, table_bytes, ids, 4ull * (uint64_t)tokens) ||
        ranges_overlap(workspace, need, grad_table, table_bytes) || ranges_overlap(workspace, need, grad_out, in_bytes) ||
        ranges_overlap(workspace, need, ids, 4ull * (uint64_t)tokens))
        return CAST_ERR_ALIAS;
    const void* ptrs[4] = {grad_out, ids, grad_table, workspace};
    if ((rc = check_device_memory(ptrs, 4)) != CAST_OK) return rc;
    SortedTokens sorted;
    if ((rc = sort_tokens(false, ids, tokens, vocab, dim, workspace, &sorted, (cudaStream_t)stream)) != CAST_OK) return rc;
    return scatter_rows(sorted, grad_out, scale, grad_table, vocab, dim, accumulate != 0, (cudaStream_t)stream);
}
