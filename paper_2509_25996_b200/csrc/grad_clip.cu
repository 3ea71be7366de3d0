// The global norm of the gradients of a model and their clipping:
//   norm = |scale| sqrt(sum over all tensors of g^2),   out = g * scale * min(1, max_norm / norm).
//
// A set of tensors is worked on as one list of tiles of kTile entries; its table travels in kernel parameter space.  One kernel walks over
// the tiles and leaves one fp64 sum per CTA; a second adds those sums, in every CTA and in the same order, and scales the tiles, the last
// ones first: part of what the first kernel read last is still in L2 (30 M fp32 gradients to bf16 45.9 us, the other way round 49.5).  Bounded by HBM: in + out, and in once more beyond L2, because the factor needs
// every gradient first.  A set that keeps its place (out = in, no conversion, factor 1) is not written.  fp32 to bf16: 109 M gradients 170 us
// (1.09 GB moved, 6.4 TB/s), 1.62 G 2.45 ms (16.2 GB, 6.6 TB/s); bf16 to bf16: 3.37 G 3.20 ms (20.2 GB, 6.3 TB/s).
//
// Squares are summed in fp32 over the 32 entries that a thread takes of a tile, and in fp64 beyond; entries whose squares leave the range of fp32
// are squared in fp64.  The factor is formed in fp64; an entry is multiplied by it in fp32 and rounded once.  The sums' order depends
// on nothing but the sizes and the device.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "bf16_access.cuh"
#include "chained.cuh"
#include "embed.cuh"

namespace cast {
namespace {

constexpr int kTile = 8192;
constexpr int kClipThreads = 256;
constexpr int kPerSm = 4;                 // CTAs; their 64 registers leave clip_kernel 416 bytes of spilled stores, which its wait for HBM covers
constexpr int kMostTensors = 1024;        // of a launch
constexpr int kFewTensors = 32;
constexpr uint64_t kSetMagic = 0x4752414453455431ull;

enum : uint8_t { kInBf16 = 1, kOutBf16 = 2, kVector = 4 };      // kVector: both aligned to 16 bytes

template <int MOST>
struct TensorTable {
    const void* in[MOST];
    void* out[MOST];
    uint64_t count[MOST];
    uint32_t start[MOST + 1];             // tiles before the tensor
    uint8_t kind[MOST];
    uint32_t n;
};

struct Span { uintptr_t lo, hi; };

struct GradSet {
    uint64_t magic;
    int device;
    bool outs;                                             // every tensor has a place for its result
    std::vector<Span> grads_at, outs_at;                   // where they lie, in the order of addresses and apart
    bool small;                                            // one table of few tensors
    TensorTable<kFewTensors> few;
    std::vector<TensorTable<kMostTensors>> tables;
};

// The tensor of a tile, from one that is at or before it.
template <int MOST>
__device__ __forceinline__ uint32_t find_tensor(const TensorTable<MOST>& t, uint32_t tile)
{
    uint32_t lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (t.start[mid] <= tile) lo = mid; else hi = mid;
    }
    return lo;
}

constexpr int kEights = kTile / 8 / kClipThreads;        // of a thread in a tile

// A thread's entries of the tile that begins at `first`, as fp32: groups of 8 neighbours, or with VEC false single ones kClipThreads apart.
// Beyond the tensor's end they are 0 and are not stored.
template <bool VEC>
__device__ __forceinline__ uint64_t entry(uint64_t first, int i, int j)
{
    return first + (VEC ? (unsigned)(i * kClipThreads + (int)threadIdx.x) * 8u + (unsigned)j : (unsigned)((i * 8 + j) * kClipThreads + (int)threadIdx.x));
}

template <bool BF16, bool VEC>
__device__ __forceinline__ void load_tile(const void* p, uint64_t first, uint64_t count, float (&v)[kEights][8])
{
#pragma unroll
    for (int i = 0; i < kEights; ++i) {
        const uint64_t at = entry<VEC>(first, i, 0);
        if (VEC && at + 8 <= count) {
            if constexpr (BF16) {
                Access<8>::unpack(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at), v[i]);
            } else {
                const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
                const float4 a = q[0], b = q[1];
                v[i][0] = a.x; v[i][1] = a.y; v[i][2] = a.z; v[i][3] = a.w; v[i][4] = b.x; v[i][5] = b.y; v[i][6] = b.z; v[i][7] = b.w;
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t one = entry<VEC>(first, i, j);
            v[i][j] = 0.0f;
            if (one < count) v[i][j] = BF16 ? bf16_low(static_cast<const uint16_t*>(p)[one]) : static_cast<const float*>(p)[one];
        }
    }
}

template <bool BF16, bool VEC>
__device__ __forceinline__ void store_tile(void* p, uint64_t first, uint64_t count, const float (&v)[kEights][8])
{
#pragma unroll
    for (int i = 0; i < kEights; ++i) {
        const uint64_t at = entry<VEC>(first, i, 0);
        if (VEC && at + 8 <= count) {
            if constexpr (BF16) {
                __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at), Access<8>::pack(v[i]));
            } else {
                float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
                __stcs(q, make_float4(v[i][0], v[i][1], v[i][2], v[i][3]));
                __stcs(q + 1, make_float4(v[i][4], v[i][5], v[i][6], v[i][7]));
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t one = entry<VEC>(first, i, j);
            if (one >= count) continue;
            if constexpr (BF16) static_cast<uint16_t*>(p)[one] = Access<1>::pack({v[i][j]});
            else static_cast<float*>(p)[one] = v[i][j];
        }
    }
}

template <bool BF16, bool VEC>
__device__ __forceinline__ double tile_squares(const void* in, uint64_t first, uint64_t count)
{
    float v[kEights][8], s = 0.0f;
    load_tile<BF16, VEC>(in, first, count, v);
#pragma unroll
    for (int i = 0; i < kEights; ++i) {
        float p = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) p = fmaf(v[i][j], v[i][j], p);
        s += p;
    }
    if (s > 0x1p-60f && s < 0x1p120f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kEights; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) d = fma((double)v[i][j], (double)v[i][j], d);
    return d;
}

// Sum over the CTA, the same bits in every thread.
__device__ __forceinline__ double cta_sum(double v)
{
    __shared__ double part[kClipThreads / 32];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < kClipThreads / 32; ++i) v += part[i];
    return v;
}

template <int MOST>
__global__ void __launch_bounds__(kClipThreads, kPerSm)
squares_kernel(const __grid_constant__ TensorTable<MOST> t, double* sums)
{
    chain_next();
    const uint32_t tiles = t.start[t.n];
    double s = 0.0;
    uint32_t i = find_tensor(t, blockIdx.x);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        while (tile >= t.start[i + 1]) ++i;
        const uint64_t first = (uint64_t)(tile - t.start[i]) * kTile;
        switch (t.kind[i] & (kInBf16 | kVector)) {
            case 0: s += tile_squares<false, false>(t.in[i], first, t.count[i]); break;
            case kInBf16: s += tile_squares<true, false>(t.in[i], first, t.count[i]); break;
            case kVector: s += tile_squares<false, true>(t.in[i], first, t.count[i]); break;
            default: s += tile_squares<true, true>(t.in[i], first, t.count[i]); break;
        }
    }
    s = cta_sum(s);
    chain_wait();
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* sums, int n, double scale)
{
    double s = 0.0;
    for (int i = (int)threadIdx.x; i < n; i += kClipThreads) s += __ldcg(sums + i);
    return fabs(scale) * sqrt(cta_sum(s));
}

__global__ void __launch_bounds__(kClipThreads)
norm_kernel(const double* sums, int n, double scale, float* norm)
{
    chain_next();
    chain_wait();
    const double v = norm_of(sums, n, scale);
    if (threadIdx.x == 0) *norm = (float)v;
}

template <bool IN, bool VEC>
__device__ __forceinline__ void scale_tile(const void* in, void* out, uint64_t first, uint64_t count, bool to_bf16, float pre, float c)
{
    float v[kEights][8];
    load_tile<IN, VEC>(in, first, count, v);
#pragma unroll
    for (int i = 0; i < kEights; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * pre * c;
    if (to_bf16) store_tile<true, VEC>(out, first, count, v);
    else store_tile<false, VEC>(out, first, count, v);
}

// `norm` may be NULL (the launches after the first).
template <int MOST>
__global__ void __launch_bounds__(kClipThreads, kPerSm)
clip_kernel(const __grid_constant__ TensorTable<MOST> t, const double* sums, int n, double scale, double max_norm, float* norm)
{
    chain_next();
    chain_wait();
    const double total = norm_of(sums, n, scale);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    // written so that a norm that is not a number makes the results that, too
    const double factor = total <= max_norm ? scale : scale * (max_norm / total);
    // a factor below the range of fp32 is taken in two steps
    const float pre = fabs(factor) < 0x1p-100 ? 0x1p-64f : 1.0f;
    const float c = (float)(factor / (double)pre);
    const uint32_t tiles = t.start[t.n];
    uint32_t i = find_tensor(t, tiles - 1 - blockIdx.x);
    for (uint32_t back = blockIdx.x; back < tiles; back += gridDim.x) {
        const uint32_t tile = tiles - 1 - back;
        while (tile < t.start[i]) --i;
        const uint8_t kind = t.kind[i];
        const void* in = t.in[i];
        void* out = t.out[i];
        if (in == out && c == 1.0f && pre == 1.0f) continue;
        const uint64_t first = (uint64_t)(tile - t.start[i]) * kTile, count = t.count[i];
        const bool to_bf16 = kind & kOutBf16;
        switch (kind & (kInBf16 | kVector)) {
            case 0: scale_tile<false, false>(in, out, first, count, to_bf16, pre, c); break;
            case kInBf16: scale_tile<true, false>(in, out, first, count, to_bf16, pre, c); break;
            case kVector: scale_tile<false, true>(in, out, first, count, to_bf16, pre, c); break;
            default: scale_tile<true, true>(in, out, first, count, to_bf16, pre, c); break;
        }
    }
}

template <int MOST>
unsigned grid_of(const TensorTable<MOST>& t, int sms)
{
    const uint32_t tiles = t.start[t.n], most = (uint32_t)(sms * kPerSm);
    return tiles < most ? tiles : most;
}

GradSet* set_of(void* p)
{
    GradSet* s = static_cast<GradSet*>(p);
    return s && s->magic == kSetMagic ? s : nullptr;
}

// The device of the set has to be the current one; its SMs, and the sums that the calls of the set leave.
int set_device(const GradSet& s, int* sms, int* n_sums)
{
    int device = 0;
    CAST_CUDA_TRY(cudaGetDevice(&device));
    if (device != s.device) return CAST_ERR_PLAN;
    CAST_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
    int n = 0;
    if (s.small) n = (int)grid_of(s.few, *sms);
    for (const auto& t : s.tables) n += (int)grid_of(t, *sms);
    *n_sums = n;
    return CAST_OK;
}

// Ranges in the order of their addresses, those that meet as one.
void join_spans(std::vector<Span>* spans)
{
    std::sort(spans->begin(), spans->end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    size_t n = 0;
    for (const Span& x : *spans) {
        if (n && x.lo <= (*spans)[n - 1].hi) (*spans)[n - 1].hi = std::max((*spans)[n - 1].hi, x.hi);
        else (*spans)[n++] = x;
    }
    spans->resize(n);
}

bool lies_in(const std::vector<Span>& spans, const void* p, uint64_t bytes)
{
    const uintptr_t lo = (uintptr_t)p, hi = lo + bytes;
    const auto behind = std::lower_bound(spans.begin(), spans.end(), hi, [](const Span& a, uintptr_t at) { return a.lo < at; });
    return behind != spans.begin() && (behind - 1)->hi > lo;
}

int check_call(GradSet* s, bool clip, float scale, const float* norm, const void* workspace, uint64_t workspace_bytes, int* sms, int* n_sums)
{
    if (!s) return CAST_ERR_PLAN;
    if (!norm || !workspace) return CAST_ERR_NULL;
    if (!std::isfinite(scale)) return CAST_ERR_HYPER;
    if (((uintptr_t)norm & 3u) || ((uintptr_t)workspace & 15u)) return CAST_ERR_ALIGN;
    int rc;
    if ((rc = set_device(*s, sms, n_sums)) != CAST_OK) return rc;
    const uint64_t need = sizeof(double) * (uint64_t)*n_sums;
    if (workspace_bytes < need) return CAST_ERR_PLAN;
    if (ranges_overlap(norm, 4, workspace, need) || lies_in(s->grads_at, norm, 4) || lies_in(s->grads_at, workspace, need)) return CAST_ERR_ALIAS;
    if (clip && (lies_in(s->outs_at, norm, 4) || lies_in(s->outs_at, workspace, need))) return CAST_ERR_ALIAS;
    const void* ptrs[2] = {norm, workspace};
    return check_device_memory(ptrs, 2);
}

int launch_squares(const GradSet& s, double* sums, int sms, cudaStream_t stream)
{
    int rc;
    if (s.small) return launch_chained(true, squares_kernel<kFewTensors>, dim3(grid_of(s.few, sms)), kClipThreads, 0, stream, 1, s.few, sums);
    bool first = true;
    for (const auto& t : s.tables) {
        const unsigned grid = grid_of(t, sms);
        if ((rc = launch_chained(first, squares_kernel<kMostTensors>, dim3(grid), kClipThreads, 0, stream, 1, t, sums)) != CAST_OK) return rc;
        first = false;
        sums += grid;
    }
    return CAST_OK;
}

template <int MOST>
void add_tensor(TensorTable<MOST>* t, const cast_grad_t& g)
{
    const uint32_t i = t->n++;
    t->in[i] = g.grad;
    t->out[i] = g.out;
    t->count[i] = (uint64_t)g.count;
    t->start[i + 1] = t->start[i] + (uint32_t)(((uint64_t)g.count + kTile - 1) / kTile);
    t->kind[i] = (uint8_t)((g.grad_bf16 ? kInBf16 : 0) | (g.out_bf16 ? kOutBf16 : 0) | (((uintptr_t)g.grad | (uintptr_t)g.out) & 15u ? 0 : kVector));
}

}  // namespace
}  // namespace cast

using namespace cast;

extern "C" int cast_grads_create(const cast_grad_t* grads, int n, void** set_out)
{
    if (!set_out) return CAST_ERR_NULL;
    *set_out = nullptr;
    if (!grads) return CAST_ERR_NULL;
    if (n < 1) return CAST_ERR_SHAPE;
    const bool outs = grads[0].out != nullptr;
    uint64_t tiles = 0;
    for (int i = 0; i < n; ++i) {
        const cast_grad_t& g = grads[i];
        if (!g.grad || (g.out != nullptr) != outs) return CAST_ERR_NULL;
        if (g.count < 1 || g.count > ((int64_t)1 << 40)) return CAST_ERR_SHAPE;
        if (((uintptr_t)g.grad & (g.grad_bf16 ? 1u : 3u)) || ((uintptr_t)g.out & (g.out_bf16 ? 1u : 3u))) return CAST_ERR_ALIGN;
        tiles += ((uint64_t)g.count + kTile - 1) / kTile;
    }
    if (tiles > 0x7FFFFFFFull) return CAST_ERR_SHAPE;
    try {
        if (outs) {
            // sorted by address, results of one another and of inputs other than their own must be apart
            struct Range { uintptr_t lo, hi; int tensor; bool out; };
            std::vector<Range> r;
            r.reserve(2 * (size_t)n);
            for (int i = 0; i < n; ++i) {
                const cast_grad_t& g = grads[i];
                const bool in_place = g.grad == g.out && !g.grad_bf16 == !g.out_bf16;
                r.push_back({(uintptr_t)g.out, (uintptr_t)g.out + (uint64_t)g.count * (g.out_bf16 ? 2u : 4u), i, true});
                if (!in_place) r.push_back({(uintptr_t)g.grad, (uintptr_t)g.grad + (uint64_t)g.count * (g.grad_bf16 ? 2u : 4u), i, false});
            }
            std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
            uintptr_t end = 0, out_end = 0;          // of everything so far, and of the results so far
            for (const Range& x : r) {
                if (x.lo < (x.out ? end : out_end)) return CAST_ERR_ALIAS;
                if (x.hi > end) end = x.hi;
                if (x.out && x.hi > out_end) out_end = x.hi;
            }
        }
        int device = 0;
        CAST_CUDA_TRY(cudaGetDevice(&device));
        for (int i = 0; i < n; ++i) {
            const void* ptrs[2] = {grads[i].grad, grads[i].out};
            for (const void* p : ptrs) {
                if (!p) continue;
                cudaPointerAttributes attr;
                CAST_CUDA_TRY(cudaPointerGetAttributes(&attr, p));
                if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged) return CAST_ERR_MEMORY;
                if (attr.type == cudaMemoryTypeDevice && attr.device != device) return CAST_ERR_MEMORY;
            }
        }
        GradSet* s = new GradSet();
        s->magic = kSetMagic;
        s->device = device;
        s->outs = outs;
        s->small = n <= kFewTensors;
        try {
            for (int i = 0; i < n; ++i) {
                const cast_grad_t& g = grads[i];
                s->grads_at.push_back({(uintptr_t)g.grad, (uintptr_t)g.grad + (uint64_t)g.count * (g.grad_bf16 ? 2u : 4u)});
                if (outs) s->outs_at.push_back({(uintptr_t)g.out, (uintptr_t)g.out + (uint64_t)g.count * (g.out_bf16 ? 2u : 4u)});
                if (s->small) {
                    add_tensor(&s->few, grads[i]);
                } else {
                    if (i % kMostTensors == 0) s->tables.emplace_back();
                    add_tensor(&s->tables.back(), grads[i]);
                }
            }
            join_spans(&s->grads_at);
            join_spans(&s->outs_at);
        } catch (...) {
            delete s;
            throw;
        }
        *set_out = s;
    } catch (...) {          // nothing but memory for the tables can fail
        return cuda_failed(cudaErrorMemoryAllocation);
    }
    return CAST_OK;
}

extern "C" int cast_grads_workspace(void* set, uint64_t* bytes)
{
    if (!bytes) return CAST_ERR_NULL;
    *bytes = 0;
    GradSet* s = set_of(set);
    if (!s) return CAST_ERR_PLAN;
    int sms = 0, n = 0, rc;
    if ((rc = set_device(*s, &sms, &n)) != CAST_OK) return rc;
    *bytes = sizeof(double) * (uint64_t)n;
    return CAST_OK;
}

extern "C" int cast_grads_norm(void* set, float scale, float* norm, void* workspace, uint64_t workspace_bytes, cast_stream_t stream)
{
    GradSet* s = set_of(set);
    int sms = 0, n = 0, rc;
    if ((rc = check_call(s, false, scale, norm, workspace, workspace_bytes, &sms, &n)) != CAST_OK) return rc;
    double* sums = static_cast<double*>(workspace);
    if ((rc = launch_squares(*s, sums, sms, (cudaStream_t)stream)) != CAST_OK) return rc;
    return launch_chained(false, norm_kernel, dim3(1), kClipThreads, 0, (cudaStream_t)stream, 1, (const double*)sums, n, (double)scale, norm);
}

extern "C" int cast_grads_clip(void* set, float max_norm, float scale, float* norm, void* workspace, uint64_t workspace_bytes, cast_stream_t stream)
{
    GradSet* s = set_of(set);
    int sms = 0, n = 0, rc;
    if (s && !s->outs) return CAST_ERR_NULL;
    if (!(max_norm >= 0.0f)) return CAST_ERR_HYPER;
    if ((rc = check_call(s, true, scale, norm, workspace, workspace_bytes, &sms, &n)) != CAST_OK) return rc;
    double* sums = static_cast<double*>(workspace);
    const cudaStream_t st = (cudaStream_t)stream;
    if ((rc = launch_squares(*s, sums, sms, st)) != CAST_OK) return rc;
    const double k = (double)scale, most = (double)max_norm;
    if (s->small) return launch_chained(false, clip_kernel<kFewTensors>, dim3(grid_of(s->few, sms)), kClipThreads, 0, st, 1, s->few, (const double*)sums, n, k, most, norm);
    for (size_t i = 0; i < s->tables.size(); ++i) {
        const auto& t = s->tables[i];
        if ((rc = launch_chained(false, clip_kernel<kMostTensors>, dim3(grid_of(t, sms)), kClipThreads, 0, st, 1, t, (const double*)sums, n, k, most,
                                 i == 0 ? norm : (float*)nullptr)) != CAST_OK)
            return rc;
    }
    return CAST_OK;
}

extern "C" int cast_grads_destroy(void* set)
{
    GradSet* s = set_of(set);
    if (!s) return CAST_ERR_PLAN;
    s->magic = 0;
    delete s;
    return CAST_OK;
}
