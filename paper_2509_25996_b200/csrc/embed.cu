// Token embedding, out[t] = scale table[ids[t]], and its gradient, grad_table[v] = scale sum_{t: ids[t] = v} grad_out[t].
//
// Forward: a gather bounded by HBM (each output row written once, each table row in use read once).  One thread moves
// 16 bytes (8 columns); kUnroll of them per thread are in flight.
//
// Gradient: the tokens are put in the order (id, position) first, so that every table row sums its tokens in one fixed
// order, in fp32 registers, and is rounded and written once, without atomics: results do not change from run to run.
//   * sort: runs of 1024 are ranked by counting (a key's place = the keys of its run that come before it, an all-pairs
//     comparison from shared memory: 1024 comparisons per key, ~1 us, no passes and no histograms), then groups of 16 runs
//     are merged at once: a key's new place = its place in its own run + its bounds in the 15 others, found by binary
//     searches that advance together, so that their loads overlap.  16384 tokens take two launches, 262144 three.
//   * sums: a row with many tokens would be one CTA's work.  Aligned pieces of kPiece sorted tokens that belong to one row
//     entirely are summed first (fp32 partial rows, one CTA each); a row then adds its head, its partial rows and its
//     tail.  Work per CTA is bounded by 2 kPiece token rows + tokens / kPiece partial rows.
#include <cmath>
#include <type_traits>

#include "embed.cuh"

namespace cast {
namespace {

constexpr int kRun = 1024;          // keys ranked by counting
constexpr int kWays = 16;           // runs merged at once
constexpr int kPiece = 64;          // sorted tokens per partial row
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
    __device__ __forceinline__ void add(const uint16_t* p, float c) {
        const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
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
    __device__ __forceinline__ void add(const uint16_t* p, float c) { v = fmaf(c, bf16_lo(__ldg(p)), v); }
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

// ------------------------------------------------------------------------------------------------ order of the tokens

constexpr int kRankThreads = 128;

__global__ void __launch_bounds__(kRankThreads)
rank_runs_kernel(const int32_t* __restrict__ ids, int32_t* __restrict__ sorted_ids, int32_t* __restrict__ order, int64_t tokens, uint32_t vocab)
{
    __shared__ uint4 keys4[kRun / 4];
    uint32_t* keys = reinterpret_cast<uint32_t*>(keys4);
    const int64_t run0 = (int64_t)(blockIdx.x / (kRun / kRankThreads)) * kRun;
    const int len = (int)min((int64_t)kRun, tokens - run0);
    const int p = (int)(blockIdx.x % (kRun / kRankThreads)) * kRankThreads + (int)threadIdx.x;
    if (p - (int)threadIdx.x >= len) return;      // uniform over the CTA
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
    if (p >= len) return;
    const uint32_t k = keys[p];
    const int own = p >> 2;
    int place = 0;
#pragma unroll 4
    for (int v = 0; v < n4; ++v) {
        const uint4 o = keys4[v];
        const uint32_t limit = k + (v < own ? 1u : 0u);      // equal keys before this one count, equal keys after it do not
        place += (o.x < limit) + (o.y < limit) + (o.z < limit) + (o.w < limit);
    }
    for (int j = 4 * own; j < p; ++j) place += keys[j] == k;
    sorted_ids[run0 + place] = (int32_t)k;
    order[run0 + place] = (int32_t)(run0 + p);
}

constexpr int kMergeThreads = 256;

// Merges groups of kWays runs of `run` keys.
__global__ void __launch_bounds__(kMergeThreads)
merge_runs_kernel(const int32_t* __restrict__ ids_in, const int32_t* __restrict__ order_in, int32_t* __restrict__ ids_out,
                  int32_t* __restrict__ order_out, int64_t tokens, int64_t run)
{
    const int64_t i = (int64_t)blockIdx.x * kMergeThreads + threadIdx.x;
    if (i >= tokens) return;
    const int64_t group0 = i / (run * kWays) * (run * kWays);
    const int own = (int)((i - group0) / run);
    const uint32_t k = (uint32_t)ids_in[i];
    uint32_t pos[kWays];
#pragma unroll
    for (int j = 0; j < kWays; ++j) pos[j] = 0u;
    for (uint32_t half = (uint32_t)run; half; half >>= 1) {
#pragma unroll
        for (int j = 0; j < kWays; ++j) {
            const int64_t start = group0 + j * run;
            const int64_t len = min(run, tokens - start);      // not positive past the last run
            const uint32_t at = pos[j] + half;
            if (j != own && (int64_t)at <= len) {
                const uint32_t limit = k + (j < own ? 1u : 0u);
                if ((uint32_t)__ldg(ids_in + start + at - 1) < limit) pos[j] = at;
            }
        }
    }
    int64_t to = group0 + (i - group0 - own * run);
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
    float* partial;               // [tokens / kPiece][dim]
    uint16_t* dest;
    int64_t tokens, vocab, dim;
    float scale;
    int lanes;                    // threads per row (a power of two)
};

template <int VEC, bool COEF>
__device__ __forceinline__ void add_tokens(Cols<VEC>& acc, const ScatterArgs& a, int64_t s, int64_t e, int64_t col)
{
#pragma unroll 4
    for (int64_t p = s; p < e; ++p) {
        const int64_t t = __ldg(a.order + p);
        acc.add(a.src + t * a.dim + col, COEF ? __ldg(a.coef + t) : 1.0f);
    }
}

// Partial rows of the aligned pieces that lie inside one table row's tokens.
template <int VEC, bool COEF>
__global__ void __launch_bounds__(kScatterThreads)
piece_sums_kernel(const __grid_constant__ ScatterArgs a)
{
    const int64_t s = (int64_t)blockIdx.x * kPiece;
    const int32_t id = a.ids[s];
    if (id != a.ids[s + kPiece - 1] || (uint32_t)id == kNoId) return;
    for (int64_t col = (int64_t)threadIdx.x * VEC; col < a.dim; col += kScatterThreads * VEC) {
        Cols<VEC> acc;
        acc.zero();
        add_tokens<VEC, COEF>(acc, a, s, s + kPiece, col);
        acc.store_partial(a.partial + (int64_t)blockIdx.x * a.dim + col);
    }
}

template <int VEC, bool COEF>
__device__ __forceinline__ void sum_row(const ScatterArgs& a, int64_t row, int64_t s, int64_t e, int lane, bool accumulate)
{
    const int64_t p0 = (s + kPiece - 1) / kPiece, p1 = e / kPiece;      // whole pieces [p0, p1)
    for (int64_t col = (int64_t)lane * VEC; col < a.dim; col += (int64_t)a.lanes * VEC) {
        Cols<VEC> acc;
        acc.zero();
        if (p0 < p1) {
            add_tokens<VEC, COEF>(acc, a, s, p0 * kPiece, col);
#pragma unroll 4
            for (int64_t p = p0; p < p1; ++p) acc.add_partial(a.partial + p * a.dim + col);
            add_tokens<VEC, COEF>(acc, a, p1 * kPiece, e, col);
        } else {
            add_tokens<VEC, COEF>(acc, a, s, e, col);
        }
        acc.store(a.dest + row * a.dim + col, a.scale, accumulate);
    }
}

// first sorted position with an id of at least `id`
__device__ __forceinline__ int64_t lower_bound(const int32_t* ids, int64_t n, int64_t id)
{
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if ((int64_t)__ldg(ids + mid) < id) lo = mid + 1; else hi = mid;
    }
    return lo;
}

constexpr int kRowsPerLaneGroup = 8;

// Every table row, the ones without a token as zeros.  A CTA takes kRowsPerLaneGroup rows per group of a.lanes threads.
template <int VEC, bool COEF>
__global__ void __launch_bounds__(kScatterThreads)
scatter_dense_kernel(const __grid_constant__ ScatterArgs a)
{
    const int groups = kScatterThreads / a.lanes;
    const int rows = groups * kRowsPerLaneGroup;
    __shared__ int64_t bound[kScatterThreads * kRowsPerLaneGroup + 1];
    const int64_t row0 = (int64_t)blockIdx.x * rows;
    for (int i = threadIdx.x; i <= rows; i += kScatterThreads) bound[i] = lower_bound(a.ids, a.tokens, min(row0 + i, a.vocab));
    __syncthreads();
    const int group = (int)threadIdx.x / a.lanes, lane = (int)threadIdx.x % a.lanes;
    for (int i = group; i < rows; i += groups)
        if (row0 + i < a.vocab) sum_row<VEC, COEF>(a, row0 + i, bound[i], bound[i + 1], lane, false);
}

// Only the rows with a token, added to what is there.  A CTA looks at kRowsPerLaneGroup sorted positions per group of
// threads; a position that begins a row's tokens does that row.
template <int VEC, bool COEF>
__global__ void __launch_bounds__(kScatterThreads)
scatter_touched_kernel(const __grid_constant__ ScatterArgs a)
{
    const int groups = kScatterThreads / a.lanes;
    const int group = (int)threadIdx.x / a.lanes, lane = (int)threadIdx.x % a.lanes;
    const int64_t first = (int64_t)blockIdx.x * groups * kRowsPerLaneGroup;
    for (int i = group; i < groups * kRowsPerLaneGroup; i += groups) {
        const int64_t p = first + i;
        if (p >= a.tokens) break;
        const int32_t id = __ldg(a.ids + p);
        if ((uint32_t)id == kNoId || (p > 0 && __ldg(a.ids + p - 1) == id)) continue;
        int64_t e = p + 1;
        if (e < a.tokens && __ldg(a.ids + e) == id) e = lower_bound(a.ids, a.tokens, (int64_t)id + 1);
        sum_row<VEC, COEF>(a, id, p, e, lane, true);
    }
}

template <int VEC, bool COEF>
int launch_scatter(const ScatterArgs& a, bool accumulate, cudaStream_t stream)
{
    if (a.tokens >= kPiece) {
        const int64_t pieces = a.tokens / kPiece;
        piece_sums_kernel<VEC, COEF><<<(unsigned)pieces, kScatterThreads, 0, stream>>>(a);
        CAST_CUDA_TRY(cudaGetLastError());
        count_launch();
    }
    const int64_t per = (int64_t)kScatterThreads / a.lanes * kRowsPerLaneGroup;
    if (accumulate) scatter_touched_kernel<VEC, COEF><<<(unsigned)((a.tokens + per - 1) / per), kScatterThreads, 0, stream>>>(a);
    else scatter_dense_kernel<VEC, COEF><<<(unsigned)((a.vocab + per - 1) / per), kScatterThreads, 0, stream>>>(a);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    return CAST_OK;
}

int64_t sort_array_bytes(int64_t tokens) { return (int64_t)align256(4ull * (uint64_t)tokens); }

}  // namespace

uint64_t scatter_scratch_bytes(int64_t tokens, int64_t dim)
{
    // two copies of (sorted ids, order), then the partial rows
    return 4ull * (uint64_t)sort_array_bytes(tokens) + align256(4ull * (uint64_t)(tokens / kPiece) * (uint64_t)dim);
}

int sort_tokens(const int32_t* ids, int64_t tokens, int64_t vocab, int64_t, void* scratch, const int32_t** sorted_ids,
                const int32_t** order, cudaStream_t stream)
{
    const int64_t step = sort_array_bytes(tokens);
    uint8_t* b = static_cast<uint8_t*>(scratch);
    int32_t* id_buf[2] = {reinterpret_cast<int32_t*>(b), reinterpret_cast<int32_t*>(b + 2 * step)};
    int32_t* or_buf[2] = {reinterpret_cast<int32_t*>(b + step), reinterpret_cast<int32_t*>(b + 3 * step)};
    const int64_t runs = (tokens + kRun - 1) / kRun;
    rank_runs_kernel<<<(unsigned)(runs * (kRun / kRankThreads)), kRankThreads, 0, stream>>>(ids, id_buf[0], or_buf[0], tokens, (uint32_t)vocab);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    int cur = 0;
    for (int64_t run = kRun; run < tokens; run *= kWays, cur ^= 1) {
        merge_runs_kernel<<<(unsigned)((tokens + kMergeThreads - 1) / kMergeThreads), kMergeThreads, 0, stream>>>(
            id_buf[cur], or_buf[cur], id_buf[cur ^ 1], or_buf[cur ^ 1], tokens, run);
        CAST_CUDA_TRY(cudaGetLastError());
        count_launch();
    }
    *sorted_ids = id_buf[cur];
    *order = or_buf[cur];
    return CAST_OK;
}

int scatter_rows(const uint16_t* src, const float* coef, float scale, const int32_t* sorted_ids, const int32_t* order, uint16_t* dest,
                 int64_t tokens, int64_t vocab, int64_t dim, bool accumulate, void* scratch, cudaStream_t stream)
{
    ScatterArgs a;
    a.src = src;
    a.coef = coef;
    a.ids = sorted_ids;
    a.order = order;
    a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + 4 * sort_array_bytes(tokens));
    a.dest = dest;
    a.tokens = tokens;
    a.vocab = vocab;
    a.dim = dim;
    a.scale = scale;
    const bool vec = dim % 8 == 0 && !((uintptr_t)src & 15u) && !((uintptr_t)dest & 15u);
    const int64_t units = vec ? dim / 8 : dim;
    a.lanes = 1;
    while (a.lanes < kScatterThreads && a.lanes < units) a.lanes *= 2;
    if (vec) return coef ? launch_scatter<8, true>(a, accumulate, stream) : launch_scatter<8, false>(a, accumulate, stream);
    return coef ? launch_scatter<1, true>(a, accumulate, stream) : launch_scatter<1, false>(a, accumulate, stream);
}

}  // namespace cast

using namespace cast;

namespace {

int check_rows(const void* a, const void* ids, const void* b, int64_t tokens, int64_t vocab, int64_t dim, float scale)
{
    if (!a || !ids || !b) return CAST_ERR_NULL;
    if (tokens < 1 || vocab < 1 || dim < 1 || tokens > 0x3FFFFFFF || vocab > 0x7FFFFFFE || dim > 0x7FFFFFFF) return CAST_ERR_SHAPE;
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
    if (tokens < 1 || dim < 1 || tokens > 0x3FFFFFFF || tokens > ((int64_t)1 << 40) / dim) return CAST_ERR_SHAPE;
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
    const int32_t *sorted, *order;
    if ((rc = sort_tokens(ids, tokens, vocab, dim, workspace, &sorted, &order, (cudaStream_t)stream)) != CAST_OK) return rc;
    return scatter_rows(grad_out, nullptr, scale, sorted, order, grad_table, tokens, vocab, dim, accumulate != 0, workspace, (cudaStream_t)stream);
}
