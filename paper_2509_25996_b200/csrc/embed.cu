// Token embedding, out[t] = scale table[ids[t]], and its gradient, grad_table[v] = scale sum_{t: ids[t] = v} grad_out[t].
//
// Forward: a gather bounded by HBM (each output row written once, each table row in use read once).  One thread moves
// 16 bytes (8 columns); kUnroll of them per thread are in flight.
//
// Gradient: the tokens are put in the order (id, position) first, so that every table row sums its tokens in one fixed
// order, in fp32 registers, and is rounded and written once, without atomics: results do not change from run to run.
//   * sort: runs of 1024 are ranked by counting (a key's place = the keys of its run that come before it, an all-pairs
//     comparison from shared memory: 1024 comparisons per key, no passes and no histograms), then groups of 16 runs
//     are merged at once: a key's new place = its place in its own run + its bounds in the 15 others, found by binary
//     searches that advance together, so that their loads overlap.  16384 tokens take two launches, 262144 three.
//   * sums: a CTA takes kPiece sorted tokens and a block of columns, asks for all of its rows at once and stores the table rows
//     whose tokens all lie in its piece.  A table row whose tokens go on in the next piece leaves fp32 partial rows (the
//     part that enters a piece and the part that leaves it), which a second kernel adds in order.  Every token row is read
//     once, and a CTA's work does not depend on how often an id occurs; only the adding of partial rows of a frequent
//     id is a chain, of tokens / kPiece rows.
//   * rows without a token: the sort is latency, not bandwidth, so the whole gradient is filled with zeros by further CTAs of
//     its kernels meanwhile.
#include <cmath>
#include <type_traits>

#include "chained.cuh"
#include "embed.cuh"

namespace cast {
namespace {

constexpr int kRun = 1024;          // keys ranked by counting
constexpr int kWays = 16;           // runs merged at once
constexpr int kPiece = 16;          // sorted tokens per CTA
constexpr uint32_t kNoId = 0x7FFFFFFFu;

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
    __device__ __forceinline__ void add_partial(const float* p) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    __device__ __forceinline__ void store_partial(float* p) const {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ void store(uint16_t* p, float scale, bool accumulate) const {
        uint4* q = reinterpret_cast<uint4*>(p);
        uint4 old = make_uint4(0u, 0u, 0u, 0u);
        if (accumulate) old = *q;
        const uint32_t o[4] = {old.x, old.y, old.z, old.w};
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack_bf16(fmaf(scale, v[2 * i], bf16_lo(o[i])), fmaf(scale, v[2 * i + 1], bf16_hi(o[i])));
        *q = make_uint4(r[0], r[1], r[2], r[3]);
    }
};
template <> struct Cols<1> {
    float v;
    __device__ __forceinline__ void zero() { v = 0.0f; }
    using Raw = uint16_t;
    static __device__ __forceinline__ Raw load(const uint16_t* p) { return __ldg(p); }
    __device__ __forceinline__ void add(Raw x, float c) { v = fmaf(c, bf16_lo(x), v); }
    __device__ __forceinline__ void add_partial(const float* p) { v += __ldg(p); }
    __device__ __forceinline__ void store_partial(float* p) const { *p = v; }
    __device__ __forceinline__ void store(uint16_t* p, float scale, bool accumulate) const {
        *p = (uint16_t)(pack_bf16(fmaf(scale, v, accumulate ? bf16_lo(*p) : 0.0f), 0.0f) & 0xFFFFu);
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

// ------------------------------------------------------------------------------------------------ zeros on the side

// A part of the gradient that CTAs [first, first + blocks) of a kernel fill with zeros.
struct Fill {
    uint16_t* dest;
    int64_t elems;
    unsigned first, blocks;
};
constexpr int64_t kFillElems = 32768;      // per CTA: 64 KB

__device__ __forceinline__ bool filled(const Fill& f)
{
    if (blockIdx.x < f.first) return false;
    const int64_t from = (int64_t)(blockIdx.x - f.first) * kFillElems, to = min(f.elems, from + kFillElems);
    if (blockIdx.y != 0) return true;
    const int64_t odd = min(to - from, (int64_t)((16u - ((uint32_t)(uintptr_t)(f.dest + from) & 15u)) & 15u) / 2);      // up to a 16-byte boundary
    const int64_t vecs = (to - from - odd) / 8;
    uint4* v = reinterpret_cast<uint4*>(f.dest + from + odd);
    for (int64_t i = threadIdx.x; i < vecs; i += blockDim.x) v[i] = make_uint4(0u, 0u, 0u, 0u);
    for (int64_t i = threadIdx.x; i < odd; i += blockDim.x) f.dest[from + i] = 0;
    for (int64_t i = from + odd + 8 * vecs + threadIdx.x; i < to; i += blockDim.x) f.dest[i] = 0;
    return true;
}

// ------------------------------------------------------------------------------------------------ order of the tokens

constexpr int kRankKeys = 128;        // keys of a run that one CTA places ...
constexpr int kRankShare = 4;         // ... with this many threads each

__global__ void __launch_bounds__(kRankKeys * kRankShare)
rank_runs_kernel(const int32_t* __restrict__ ids, int32_t* __restrict__ sorted_ids, int32_t* __restrict__ order, int64_t tokens, uint32_t vocab,
                 const __grid_constant__ Fill fill)
{
    __shared__ uint4 keys4[kRun / 4];
    uint32_t* keys = reinterpret_cast<uint32_t*>(keys4);
    chain_next();
    if (filled(fill)) return;
    chain_wait();
    const int64_t run0 = (int64_t)(blockIdx.x / (kRun / kRankKeys)) * kRun;
    const int len = (int)min((int64_t)kRun, tokens - run0);
    const int first = (int)(blockIdx.x % (kRun / kRankKeys)) * kRankKeys;
    if (first >= len) return;             // uniform over the CTA
    const int n4 = (len + 3) / 4;
    for (int i = threadIdx.x; i < 4 * n4; i += kRankKeys * kRankShare) {
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
        sorted_ids[run0 + place] = (int32_t)k;
        order[run0 + place] = (int32_t)(run0 + p);
    }
}

constexpr int kMergeThreads = 128;

// Merges groups of kWays runs of `run` keys.  The searches of a key advance together and without branches: kWays
// independent loads per halving.
__global__ void __launch_bounds__(kMergeThreads)
merge_runs_kernel(const int32_t* __restrict__ ids_in, const int32_t* __restrict__ order_in, int32_t* __restrict__ ids_out,
                  int32_t* __restrict__ order_out, int32_t tokens, int32_t run, const __grid_constant__ Fill fill)
{
    chain_next();
    if (filled(fill)) return;
    chain_wait();
    const int32_t i = (int32_t)blockIdx.x * kMergeThreads + (int32_t)threadIdx.x;
    if (i >= tokens) return;
    const int64_t group = (int64_t)run * kWays;
    const int32_t group0 = (int32_t)(i / group * group);
    const int own = (i - group0) / run;
    const uint32_t k = (uint32_t)ids_in[i];
    const int32_t left = tokens - group0;            // keys of the group, and of the groups after it
    int32_t pos[kWays];
#pragma unroll
    for (int j = 0; j < kWays; ++j) pos[j] = 0;
    for (int32_t half = run; half; half >>= 1) {
#pragma unroll
        for (int j = 0; j < kWays; ++j) {
            const int64_t before = (int64_t)j * run;                 // keys of the group ahead of run j
            const int32_t at = pos[j] + half;
            const bool there = at <= run && before + at <= left;
            const uint32_t limit = j == own ? 0u : k + (j < own ? 1u : 0u);
            const uint32_t other = (uint32_t)__ldg(ids_in + group0 + (there ? (int32_t)before + at - 1 : 0));
            pos[j] = there && other < limit ? at : pos[j];
        }
    }
    int64_t to = (int64_t)group0 + (i - group0 - own * run);
#pragma unroll
    for (int j = 0; j < kWays; ++j) to += pos[j];
    ids_out[to] = (int32_t)k;
    order_out[to] = order_in[i];
}

// ------------------------------------------------------------------------------------------------ sums

constexpr int kScatterThreads = 256;

struct ScatterArgs {
    const uint16_t* src;
    const float* coef;            // per token, or nullptr
    const int32_t* ids;           // sorted
    const int32_t* order;
    float* partial;               // [pieces][2][dim]: what enters a piece, what leaves it
    uint16_t* dest;
    int64_t dim;
    int32_t tokens, pieces;
    float scale;
    int lanes;                    // threads per row: 32 .. 256, a power of two
    int accumulate;
};

// Column of this thread: a.lanes threads per row, the rest of a long row in blockIdx.y.
template <int VEC>
__device__ __forceinline__ int32_t column_of(const ScatterArgs& a)
{
    return ((int32_t)blockIdx.y * a.lanes + (int)threadIdx.x % a.lanes) * VEC;
}

// One piece of kPiece sorted tokens per group of a.lanes threads.
template <int VEC, bool COEF>
__global__ void __launch_bounds__(kScatterThreads, 3)
piece_sums_kernel(const __grid_constant__ ScatterArgs a)
{
    constexpr int kBatch = 8;             // token rows asked for at a time
    chain_next();
    chain_wait();
    const int32_t piece = (int32_t)blockIdx.x * (kScatterThreads / a.lanes) + (int)threadIdx.x / a.lanes;
    if (piece >= a.pieces) return;
    const int32_t col = column_of<VEC>(a);
    if (col >= a.dim) return;
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
    for (int i = 0; i < kPiece; ++i) t[i] = i < n && id[i + 1] != kNoId ? __ldg(a.order + p0 + i) : -1;
    const uint16_t* src = a.src + col;
    float* partial = a.partial + (int64_t)piece * 2 * a.dim + col;
    bool entered = id[0] == id[1];        // the current row's tokens began in an earlier piece
    Cols<VEC> acc;
    acc.zero();
#pragma unroll
    for (int b = 0; b < kPiece; b += kBatch) {
        typename Cols<VEC>::Raw x[kBatch];
        float c[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            c[i] = 1.0f;
            if (t[b + i] >= 0) {
                x[i] = Cols<VEC>::load(src + (int64_t)t[b + i] * a.dim);
                if constexpr (COEF) c[i] = __ldg(a.coef + t[b + i]);
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (t[b + i] < 0) continue;
            acc.add(x[i], c[i]);
            const uint32_t own = id[b + i + 1];
            if (id[b + i + 2] != own) {                    // its last token
                if (entered) acc.store_partial(partial);
                else acc.store(a.dest + (int64_t)own * a.dim + col, a.scale, a.accumulate);
                entered = false;
                acc.zero();
            } else if (b + i == kPiece - 1) {              // goes on in the next piece
                acc.store_partial(entered ? partial : partial + a.dim);
            }
        }
    }
}

// End of the positions after p that hold the id at p.  All lanes of a warp ask for the same p: 32 positions per load.
__device__ __forceinline__ int32_t end_of(const int32_t* ids, int32_t n, int32_t p, int32_t id)
{
    const int lane = (int)threadIdx.x & 31;
    int32_t lo = p + 1, step = 1;                          // [p, lo) hold it
    for (;;) {                                             // strides of 1, 32, 1024, ... positions until one ends it
        const int64_t at = (int64_t)lo + (int64_t)(lane + 1) * step - 1;
        const int same = __popc(__ballot_sync(0xFFFFFFFFu, at < n && __ldg(ids + at) == id));
        lo += same * step;
        if (same < 32) break;
        step *= 32;
    }
    while (step > 1) {                                     // then 32 times finer inside the stride that did
        step /= 32;
        const int64_t at = (int64_t)lo + (int64_t)(lane + 1) * step - 1;
        lo += __popc(__ballot_sync(0xFFFFFFFFu, at < n && __ldg(ids + at) == id)) * step;
    }
    return lo;
}

// The table rows that leave a piece they began in: what left it, then what entered the pieces after it.
template <int VEC>
__global__ void __launch_bounds__(kScatterThreads)
join_pieces_kernel(const __grid_constant__ ScatterArgs a)
{
    chain_next();
    chain_wait();
    const int32_t piece = (int32_t)blockIdx.x * (kScatterThreads / a.lanes) + (int)threadIdx.x / a.lanes;
    const int32_t p0 = piece * kPiece, last = p0 + kPiece - 1;
    if (piece + 1 >= a.pieces) return;                     // the last piece: nothing leaves it
    const int32_t id = __ldg(a.ids + last);
    if ((uint32_t)id == kNoId || __ldg(a.ids + last + 1) != id || (p0 > 0 && __ldg(a.ids + p0 - 1) == id)) return;
    const int32_t e = end_of(a.ids, a.tokens, last, id);
    const int32_t col = column_of<VEC>(a);
    if (col >= a.dim) return;
    Cols<VEC> acc;
    acc.zero();
    const float* p = a.partial + (int64_t)piece * 2 * a.dim + col;
    acc.add_partial(p + a.dim);
    const int32_t count = (e - 1) / kPiece - piece;
#pragma unroll 8
    for (int32_t i = 0; i < count; ++i) {
        p += 2 * a.dim;
        acc.add_partial(p);
    }
    acc.store(a.dest + (int64_t)id * a.dim + col, a.scale, a.accumulate);
}

// Part `i` of `n` equal parts of a gradient, whole CTAs of zeros each.
Fill fill_part(uint16_t* dest, int64_t elems, int i, int n, unsigned first)
{
    const int64_t blocks = (elems + kFillElems - 1) / kFillElems, from = blocks * i / n, to = blocks * (i + 1) / n;
    const int64_t start = from * kFillElems, stop = to * kFillElems < elems ? to * kFillElems : elems;
    return {dest + start, stop - start, first, (unsigned)(to - from)};
}

template <int VEC, bool COEF>
int launch_scatter(const ScatterArgs& a, cudaStream_t stream)
{
    const int64_t units = (a.dim + VEC - 1) / VEC, groups = kScatterThreads / a.lanes;
    const dim3 grid((unsigned)((a.pieces + groups - 1) / groups), (unsigned)((units + a.lanes - 1) / a.lanes));
    const int rc = launch_chained(false, piece_sums_kernel<VEC, COEF>, grid, kScatterThreads, 0, stream, 1, a);
    if (rc != CAST_OK || a.pieces < 2) return rc;
    return launch_chained(false, join_pieces_kernel<VEC>, grid, kScatterThreads, 0, stream, 1, a);
}

int64_t sort_array_bytes(int64_t tokens) { return (int64_t)align256(4ull * (uint64_t)tokens); }

}  // namespace

uint64_t scatter_scratch_bytes(int64_t tokens, int64_t dim)
{
    // two copies of (sorted ids, order), then the partial rows
    return 4ull * (uint64_t)sort_array_bytes(tokens) + align256(8ull * (uint64_t)((tokens + kPiece - 1) / kPiece) * (uint64_t)dim);
}

int sort_tokens(bool first, const int32_t* ids, int64_t tokens, int64_t vocab, int64_t dim, void* scratch, uint16_t* zeros, SortedTokens* sorted,
                cudaStream_t stream)
{
    const int64_t step = sort_array_bytes(tokens);
    uint8_t* b = static_cast<uint8_t*>(scratch);
    int32_t* id_buf[2] = {reinterpret_cast<int32_t*>(b), reinterpret_cast<int32_t*>(b + 2 * step)};
    int32_t* or_buf[2] = {reinterpret_cast<int32_t*>(b + step), reinterpret_cast<int32_t*>(b + 3 * step)};
    int kernels = 1, done = 0;            // that share the filling: the ranking and the merges
    for (int64_t run = kRun; run < tokens; run *= kWays) ++kernels;
    auto part = [&](unsigned own) {
        const Fill f = zeros ? fill_part(zeros, vocab * dim, done, kernels, own) : Fill{nullptr, 0, own, 0};
        ++done;
        return f;
    };
    const unsigned rank_blocks = (unsigned)((tokens + kRun - 1) / kRun * (kRun / kRankKeys));
    Fill f = part(rank_blocks);
    int rc = launch_chained(first, rank_runs_kernel, dim3(rank_blocks + f.blocks), kRankKeys * kRankShare, 0, stream, 1, ids, id_buf[0], or_buf[0], tokens,
                            (uint32_t)vocab, f);
    if (rc != CAST_OK) return rc;
    int cur = 0;
    for (int64_t run = kRun; run < tokens; run *= kWays, cur ^= 1) {
        const unsigned own = (unsigned)((tokens + kMergeThreads - 1) / kMergeThreads);
        f = part(own);
        rc = launch_chained(false, merge_runs_kernel, dim3(own + f.blocks), kMergeThreads, 0, stream, 1, id_buf[cur], or_buf[cur], id_buf[cur ^ 1],
                            or_buf[cur ^ 1], (int32_t)tokens, (int32_t)run, f);
        if (rc != CAST_OK) return rc;
    }
    sorted->ids = id_buf[cur];
    sorted->order = or_buf[cur];
    sorted->scratch = b + 4 * step;
    sorted->tokens = tokens;
    return CAST_OK;
}

int scatter_rows(const SortedTokens& sorted, const uint16_t* src, const float* coef, float scale, uint16_t* dest, int64_t dim,
                 bool accumulate, cudaStream_t stream)
{
    ScatterArgs a;
    a.src = src;
    a.coef = coef;
    a.ids = sorted.ids;
    a.order = sorted.order;
    a.partial = static_cast<float*>(sorted.scratch);
    a.dest = dest;
    a.tokens = (int32_t)sorted.tokens;
    a.pieces = (int32_t)((sorted.tokens + kPiece - 1) / kPiece);
    a.dim = dim;
    a.scale = scale;
    a.accumulate = accumulate;
    const bool vec = dim % 8 == 0 && !((uintptr_t)src & 15u) && !((uintptr_t)dest & 15u);
    const int64_t units = vec ? dim / 8 : dim;
    a.lanes = 32;
    while (a.lanes < kScatterThreads && a.lanes < units) a.lanes *= 2;
    if (vec) return coef ? launch_scatter<8, true>(a, stream) : launch_scatter<8, false>(a, stream);
    return coef ? launch_scatter<1, true>(a, stream) : launch_scatter<1, false>(a, stream);
}

}  // namespace cast

using namespace cast;

namespace {

constexpr int64_t kMostColumns = 1 << 23;      // blocks of 256 accesses of one column each: fewer than 2^16

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
    if ((rc = sort_tokens(true, ids, tokens, vocab, dim, workspace, accumulate ? nullptr : grad_table, &sorted, (cudaStream_t)stream)) != CAST_OK) return rc;
    return scatter_rows(sorted, grad_out, nullptr, scale, grad_table, dim, accumulate != 0, (cudaStream_t)stream);
}
