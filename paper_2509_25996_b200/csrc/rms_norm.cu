// Root-mean-square norm of the rows of a residual stream, and its gradient.
//
//   forward    h = bf16(x + residual) (or h = x),  r = 1 / sqrt(mean(h^2) + eps),  y = weight h r
//   gradient   n = h r,  g = weight dy,  dx = r (g - n mean(g n)) + dh,  dweight = sum over the rows of dy n
//
// Forward: one pass; a row stays in registers between its sum of squares and its result.  `lanes` threads share a row, each with up to
// N accesses of W columns: 8 to 32 lanes of a warp (several rows per warp or CTA, no barrier), or a whole CTA.  Bounded by HBM.
//
// Gradient: the statistics of a row come from h again instead of being kept (one more multiply-add per column, 4 bytes per row less, nothing to
// pass on).  CTAs walk over rows with a stride; a thread owns the same columns of all of its rows and sums their part of
// dweight in registers.  The next row is asked for before the current one is worked on.  Each CTA leaves one fp32
// row of sums, and a second kernel adds those: no atomics, the same bits every time.
//
// Roundings: sums and statistics are fp32 (fp64 for rows whose squares leave the range of fp32), y and dx are rounded once; h is rounded to
// bf16 first, because that is the stream that is stored and normalised again by the backward pass.
#include <cmath>
#include <type_traits>

#include "bf16_access.cuh"
#include "chained.cuh"
#include "embed.cuh"

namespace cast {
namespace {

constexpr int64_t kMostColumns = 32768;      // 1024 threads x 4 accesses of 8 columns, or x 32 of one
constexpr int kGroup = 32;                   // columns that share a scale in the 8-bit form
constexpr int kMostWarps = 32;

struct NormArgs {
    const uint16_t* x;
    const uint16_t* residual;
    const void* weight;
    uint16_t* y;              // bf16 result, or
    uint8_t* q;               // e4m3 result and
    uint8_t* scales;          // its scales, powers of two
    uint16_t* h;
    int32_t tokens;
    int32_t dim;
    int32_t units;            // accesses of a row
    int32_t lanes;            // threads of a row
    float eps;
};

// Sum over the `lanes` threads of a row (all of the CTA with SPLIT); every one of them gets it, summed in the same order.
template <bool SPLIT, class T>
__device__ __forceinline__ T row_sum(T v, int lanes, T* shared)
{
    const int width = SPLIT ? 32 : lanes;
    for (int d = width >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if constexpr (SPLIT) {
        if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
        __syncthreads();
        const int warps = (int)blockDim.x >> 5;
        v = shared[0];
        for (int i = 1; i < warps; ++i) v += shared[i];
    }
    return v;
}

// Squares of such rows over- or underflow in fp32 (mean: of the squares; NaN, too).
__device__ __forceinline__ bool odd_row(float mean_eps) { return !(mean_eps < 0x1p100f && mean_eps > 0x1p-100f); }
// A power of two that brings the entries of such a row back into the range: 1/sqrt(mean) = pre * (1/sqrt(mean) / pre).
__device__ __forceinline__ float odd_factor(double mean_eps) { return mean_eps < 1.0 ? 0x1p64f : 0x1p-64f; }

// Two e4m3 values, the first in the low byte; beyond +-448 only by a rounding, NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// The scale of a group whose largest magnitude has the bits `top`: the least power of two s with top <= 448 s, as its exponent + 127
// (0 for zeros, 255 = NaN where an entry is not finite).  448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t group_scale(uint32_t top)
{
    const int e = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return top >= 0x7F800000u ? 255u : (uint32_t)max(e, 0);
}
// 1 / scale, exact
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float(s == 255u ? 0x7FC00000u : (254u - s) << 23); }

template <int W, int N, bool SPLIT, bool RES, bool MX, class WT>
__global__ void __launch_bounds__(SPLIT ? 1024 : 256)
rms_norm_kernel(const __grid_constant__ NormArgs a)
{
    using A = Access<W>;
    using Raw = typename A::Raw;
    __shared__ float part[kMostWarps];
    __shared__ double part64[kMostWarps];
    const int lane = SPLIT ? (int)threadIdx.x : (int)threadIdx.x & (a.lanes - 1);
    const int64_t row = SPLIT ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / a.lanes) + threadIdx.x / a.lanes;
    const bool active = SPLIT || row < a.tokens;
    const int64_t base = row * a.dim;
    Raw h[N];
    if constexpr (RES) {
        Raw r[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            h[i] = r[i] = A::zero();
            if (active && c < a.units) {
                h[i] = *reinterpret_cast<const Raw*>(a.x + base + (int64_t)c * W);
                r[i] = *reinterpret_cast<const Raw*>(a.residual + base + (int64_t)c * W);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            float u[W], v[W];
            A::unpack(h[i], u);
            A::unpack(r[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) u[j] += v[j];
            h[i] = A::pack(u);
            if (active && c < a.units) *reinterpret_cast<Raw*>(a.h + base + (int64_t)c * W) = h[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            h[i] = A::zero();
            if (active && c < a.units) h[i] = *reinterpret_cast<const Raw*>(a.x + base + (int64_t)c * W);
        }
    }
    float square = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[W];
        A::unpack(h[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j) square = fmaf(v[j], v[j], square);
    }
    const float mean = row_sum<SPLIT>(square, a.lanes, part) / (float)a.dim + a.eps;
    float r = __frsqrt_rn(mean), pre = 1.0f;
    if (SPLIT ? odd_row(mean) : __any_sync(0xFFFFFFFFu, odd_row(mean))) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[W];
            A::unpack(h[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) s = fma((double)v[j], (double)v[j], s);
        }
        s = row_sum<SPLIT>(s, a.lanes, part64) / (double)a.dim + (double)a.eps;
        if (odd_row(mean)) {
            pre = odd_factor(s);
            r = (float)(1.0 / sqrt(s) / (double)pre);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = i * a.lanes + lane;
        const bool in = active && c < a.units;
        float v[W], w[W];
        A::unpack(h[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = 0.0f;
        if (in) A::weights(static_cast<const WT*>(a.weight) + c * W, w);
        // two bf16 entries multiply exactly: one rounding less than the other way round
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = v[j] * pre * w[j] * r;
        if constexpr (!MX) {
            if (in) *reinterpret_cast<Raw*>(a.y + base + (int64_t)c * W) = A::pack(v);
        } else {
            // a group is 4 neighbouring lanes of 8 columns, or a warp of one column each; magnitudes are compared as integers, so that NaN
            // counts as the largest
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < W; ++j) top = max(top, __float_as_uint(in ? v[j] : 0.0f) & 0x7FFFFFFFu);
#pragma unroll
            for (int d = kGroup / W / 2; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            const uint32_t s = group_scale(top);
            const float inv = inverse_scale(s);
            if (!in) continue;
            if constexpr (W == 8) {
                *reinterpret_cast<uint2*>(a.q + base + (int64_t)c * W) =
                    make_uint2(e4m3_pair(v[0] * inv, v[1] * inv) | e4m3_pair(v[2] * inv, v[3] * inv) << 16,
                               e4m3_pair(v[4] * inv, v[5] * inv) | e4m3_pair(v[6] * inv, v[7] * inv) << 16);
            } else {
                a.q[base + c] = (uint8_t)e4m3_pair(v[0] * inv, 0.0f);
            }
            if (c % (kGroup / W) == 0) a.scales[row * ((a.dim + kGroup - 1) / kGroup) + c / (kGroup / W)] = (uint8_t)s;
        }
    }
}

// How a row is spread: lanes and accesses per lane (N, one of the instantiated ones); lanes <= 32 are lanes of one warp.
struct Spread {
    int lanes, n;
    bool split;
};

Spread spread_of(int64_t units, int w)
{
    if (w == 8) {
        if (units <= 128) {                   // up to 1024 columns: in a warp
            int lanes = 8;
            while (lanes < 32 && lanes < units) lanes *= 2;
            const int n = (int)((units + lanes - 1) / lanes);
            return {lanes, n <= 1 ? 1 : n <= 2 ? 2 : 4, false};
        }
        const int n = units <= 512 ? 1 : units <= 2048 ? 2 : 4;
        return {(int)((units + n * 32 - 1) / (n * 32)) * 32, n, true};
    }
    if (units <= 256) return {32, 8, false};
    const int n = units <= 8192 ? 8 : 32;
    return {(int)((units + n * 32 - 1) / (n * 32)) * 32, n, true};
}

template <int W, int N, bool SPLIT, bool RES, bool MX, class WT>
int launch_norm(const NormArgs& a, cudaStream_t stream)
{
    const unsigned threads = SPLIT ? (unsigned)a.lanes : 256u;
    const unsigned rows = SPLIT ? 1u : threads / (unsigned)a.lanes;
    rms_norm_kernel<W, N, SPLIT, RES, MX, WT><<<((unsigned)a.tokens + rows - 1) / rows, threads, 0, stream>>>(a);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    return CAST_OK;
}

template <int W, int N, bool SPLIT>
int launch_norm(const NormArgs& a, bool weight_fp32, cudaStream_t stream)
{
    if (a.residual) {
        if (a.q) return weight_fp32 ? launch_norm<W, N, SPLIT, true, true, float>(a, stream) : launch_norm<W, N, SPLIT, true, true, uint16_t>(a, stream);
        return weight_fp32 ? launch_norm<W, N, SPLIT, true, false, float>(a, stream) : launch_norm<W, N, SPLIT, true, false, uint16_t>(a, stream);
    }
    if (a.q) return weight_fp32 ? launch_norm<W, N, SPLIT, false, true, float>(a, stream) : launch_norm<W, N, SPLIT, false, true, uint16_t>(a, stream);
    return weight_fp32 ? launch_norm<W, N, SPLIT, false, false, float>(a, stream) : launch_norm<W, N, SPLIT, false, false, uint16_t>(a, stream);
}

// ------------------------------------------------------------------------------------------------ gradient

struct NormGradArgs {
    const uint16_t* dy;
    const uint16_t* h;
    const uint16_t* dh;       // or NULL
    const void* weight;
    uint16_t* dx;
    float* partial;           // [grid][dim], or NULL: no gradient of the weight
    int32_t tokens;
    int32_t dim;
    int32_t units;
    int32_t lanes;
    float eps;
};

// The rows of a CTA pass through a ring of kStages rows' worth of its threads' own accesses: with 16-byte accesses the copies go to shared
// memory without waiting (cp.async: a thread reads only what it copied itself, so no barrier is needed), one access of one
// column goes through registers, when its row's turn comes.
__device__ __forceinline__ void copy_async(uint4* shared, const void* global, bool in)
{
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(shared);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(global), "r"(in ? 16 : 0) : "memory");      // zeros where not `in`
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(PENDING) : "memory"); }

// Entries of one access of the row that is being worked on.
template <int W, int N, int STAGES, bool RES>
struct GradRow {
    using A = Access<W>;
    using Raw = typename A::Raw;
    static constexpr int kArrays = RES ? 3 : 2;
    Raw held[W == 8 ? 1 : kArrays * N];             // W == 1: the row's accesses
    uint4* ring;                                     // W == 8: [STAGES][kArrays][N][threads]

    static __device__ __forceinline__ const uint16_t* source(const NormGradArgs& a, int k) { return k == 0 ? a.h : k == 1 ? a.dy : a.dh; }
    __device__ __forceinline__ void fetch(const NormGradArgs& a, int64_t row, int lane, int stage)
    {
        if constexpr (W == 8) {
#pragma unroll
            for (int k = 0; k < kArrays; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = i * a.lanes + lane;
                    const bool in = row < a.tokens && c < a.units;
                    copy_async(ring + ((stage * kArrays + k) * N + i) * (int)blockDim.x + (int)threadIdx.x, source(a, k) + (in ? row * a.dim + c * 8 : 0), in);
                }
            copies_commit();
        } else {
#pragma unroll
            for (int k = 0; k < kArrays; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = i * a.lanes + lane;
                    held[k * N + i] = A::zero();
                    if (row < a.tokens && c < a.units) held[k * N + i] = source(a, k)[row * a.dim + c];
                }
        }
    }
    __device__ __forceinline__ void get(int k, int i, int stage, float (&v)[W]) const
    {
        if constexpr (W == 8) A::unpack(ring[((stage * kArrays + k) * N + i) * (int)blockDim.x + (int)threadIdx.x], v);
        else A::unpack(held[k * N + i], v);
    }
};

template <int W, int N, int STAGES, bool SPLIT, bool RES, class WT>
__global__ void __launch_bounds__(SPLIT ? (W * N <= 16 ? 512 : 1024) : 256, SPLIT && W * N > 8 ? 1 : 2)
rms_norm_grad_kernel(const __grid_constant__ NormGradArgs a)
{
    using A = Access<W>;
    extern __shared__ uint4 dynamic[];               // the ring; !SPLIT, afterwards: [rows of the CTA][dim] sums
    __shared__ float2 part[2][kMostWarps];
    __shared__ double part64[2][kMostWarps];
    const int lane = SPLIT ? (int)threadIdx.x : (int)threadIdx.x & (a.lanes - 1);
    const int rows = SPLIT ? 1 : (int)blockDim.x / a.lanes, sub = SPLIT ? 0 : (int)threadIdx.x / a.lanes;
    float dw[N][W];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) dw[i][j] = 0.0f;
    auto weight = [&](int i, float (&w)[W]) {
        const int c = i * a.lanes + lane;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = 0.0f;
        if (c < a.units) A::weights(static_cast<const WT*>(a.weight) + c * W, w);
    };
    constexpr bool KEPT = W * N <= 16;                // the weights of a thread's columns in registers
    float kept[KEPT ? N : 1][W];
    if constexpr (KEPT) {
#pragma unroll
        for (int i = 0; i < N; ++i) weight(i, kept[i]);
    }
    const int64_t step = (int64_t)gridDim.x * rows;
    int64_t row0 = (int64_t)blockIdx.x * rows;
    GradRow<W, N, STAGES, RES> x;
    x.ring = dynamic;
    if constexpr (W == 8) {
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) x.fetch(a, row0 + sub + k * step, lane, k);
    }
    int stage = 0;
    for (int turn = 0; row0 < a.tokens; row0 += step, turn ^= 1, stage = stage + 1 == STAGES ? 0 : stage + 1) {
        const int64_t row = row0 + sub;
        x.fetch(a, row + (W == 8 ? (STAGES - 1) * step : 0), lane, W == 8 ? (stage + STAGES - 1) % STAGES : 0);
        if constexpr (W == 8) copies_wait<STAGES - 1>();
        float2 s = make_float2(0.0f, 0.0f);          // sums of h^2 and of g h
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float u[W], v[W], w[W];
            x.get(0, i, stage, u);
            x.get(1, i, stage, v);
            if constexpr (!KEPT) weight(i, w);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                s.x = fmaf(u[j], u[j], s.x);
                s.y = fmaf(v[j] * (KEPT ? kept[KEPT ? i : 0][j] : w[j]), u[j], s.y);
            }
        }
        for (int d = (SPLIT ? 32 : a.lanes) >> 1; d > 0; d >>= 1) {
            s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, d);
            s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, d);
        }
        if constexpr (SPLIT) {
            // two buffers: a warp may be one row ahead of another, not two
            if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = s;
            __syncthreads();
            s = part[turn][0];
            for (int i = 1; i < (int)(blockDim.x >> 5); ++i) {
                const float2 o = part[turn][i];
                s.x += o.x;
                s.y += o.y;
            }
        }
        const float mean = s.x / (float)a.dim + a.eps;
        float r = __frsqrt_rn(mean), pre = 1.0f, scaled = r;             // r = pre * scaled
        float m = s.y / (float)a.dim * r;                               // mean(g n)
        if (SPLIT ? odd_row(mean) : __any_sync(0xFFFFFFFFu, odd_row(mean))) {
            double s64 = 0.0, m64 = 0.0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float u[W], v[W], w[W];
                x.get(0, i, stage, u);
                x.get(1, i, stage, v);
                weight(i, w);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    s64 = fma((double)u[j], (double)u[j], s64);
                    m64 = fma((double)v[j] * (double)w[j], (double)u[j], m64);
                }
            }
            if constexpr (SPLIT) __syncthreads();                        // the row before may have been an odd one, too
            s64 = row_sum<SPLIT>(s64, a.lanes, part64[0]) / (double)a.dim + (double)a.eps;
            m64 = row_sum<SPLIT>(m64, a.lanes, part64[1]) / (double)a.dim;
            if (odd_row(mean)) {
                const double r64 = 1.0 / sqrt(s64);
                pre = odd_factor(s64);
                scaled = (float)(r64 / (double)pre);
                r = (float)r64;
                m = (float)(m64 * r64);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            if (row >= a.tokens || c >= a.units) continue;
            float u[W], v[W], w[W], o[W];
            x.get(0, i, stage, u);
            x.get(1, i, stage, v);
            if constexpr (!KEPT) weight(i, w);
            if constexpr (RES) x.get(2, i, stage, o);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float n = u[j] * pre * scaled;
                dw[i][j] = fmaf(v[j], n, dw[i][j]);
                const float d = fmaf(v[j], KEPT ? kept[KEPT ? i : 0][j] : w[j], -n * m);
                o[j] = RES ? fmaf(r, d, o[j]) : r * d;
            }
            *reinterpret_cast<typename A::Raw*>(a.dx + row * a.dim + (int64_t)c * W) = A::pack(o);
        }
    }
    chain_next();
    if constexpr (W == 8) copies_wait<0>();
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.x * a.dim;
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            if (c >= a.units) continue;
            if constexpr (W == 8) {
                float4* q = reinterpret_cast<float4*>(out + c * 8);
                q[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
                q[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
            } else {
                out[c] = dw[i][0];
            }
        }
    } else {
        float* sums = reinterpret_cast<float*>(dynamic);
        __syncthreads();                             // the ring has been read
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            if (c >= a.units) continue;
#pragma unroll
            for (int j = 0; j < W; ++j) sums[sub * a.dim + c * W + j] = dw[i][j];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.dim; c += blockDim.x) {
            float v = sums[c];
            for (int i = 1; i < rows; ++i) v += sums[i * a.dim + c];
            out[c] = v;
        }
    }
}

// dweight[c] = sum of `rows` partial rows: 32 columns per CTA, its warps share the rows.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps)
join_weight_grad_kernel(const float* partial, float* out, int32_t rows, int32_t dim)
{
    __shared__ float sums[kJoinWarps][33];
    chain_next();
    chain_wait();
    const int lane = (int)threadIdx.x & 31, warp = (int)threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (c < dim) {
#pragma unroll 8
        for (int r = warp; r < rows; r += kJoinWarps) v += __ldcg(partial + (int64_t)r * dim + c);
    }
    sums[warp][lane] = v;
    __syncthreads();
    v = sums[lane][warp];                            // warp w adds up column w
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int64_t own = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && own < dim) out[own] = v;
}

struct GradSpread {
    Spread s;
    int stages;
};

GradSpread grad_spread_of(int64_t units, int w)
{
    if (w == 8) {
        if (units <= 128) {                   // up to 1024 columns: in a warp
            int lanes = 8;
            while (lanes < 32 && lanes < units) lanes *= 2;
            const int n = (int)((units + lanes - 1) / lanes);
            return {{lanes, n <= 1 ? 1 : n <= 2 ? 2 : 4, false}, n <= 2 ? 4 : 2};
        }
        // stages of 48 bytes for each access: 96 KB a CTA (two of them on an SM), 192 KB for wider rows (one)
        const int n = units <= 512 ? 1 : units <= 1024 ? 2 : 4;
        return {{(int)((units + n * 32 - 1) / (n * 32)) * 32, n, true}, units <= 1024 ? 4 : units <= 2048 ? 2 : 1};
    }
    if (units <= 256) return {{32, 8, false}, 1};
    const int n = units <= 4096 ? 8 : 32;
    return {{(int)((units + n * 32 - 1) / (n * 32)) * 32, n, true}, 1};
}

int sm_count(int* sms)
{
    int device = 0;
    CAST_CUDA_TRY(cudaGetDevice(&device));
    CAST_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
    return CAST_OK;
}

// CTAs of the gradient kernel: what the SMs hold at a time, and no more than there are groups of rows.
int64_t grad_ctas(const Spread& s, int64_t tokens, int sms)
{
    const int64_t rows = s.split ? 1 : 256 / s.lanes, groups = (tokens + rows - 1) / rows;
    const int64_t held = (int64_t)sms * (s.split && s.n * s.lanes > 512 ? 1 : 2);
    return groups < held ? groups : held;
}

// Workspace for either width of access: which one a call takes depends on its pointers.
uint64_t grad_workspace(int64_t tokens, int64_t dim, int sms)
{
    const int64_t wide = dim % 8 == 0 ? grad_ctas(grad_spread_of(dim / 8, 8).s, tokens, sms) : 0, one = grad_ctas(grad_spread_of(dim, 1).s, tokens, sms);
    return sizeof(float) * (uint64_t)(wide > one ? wide : one) * (uint64_t)dim;
}

template <int W, int N, int STAGES, bool SPLIT, bool RES, class WT>
int launch_grad(const NormGradArgs& a, unsigned ctas, cudaStream_t stream)
{
    const unsigned threads = SPLIT ? (unsigned)a.lanes : 256u;
    const size_t ring = W == 8 ? (size_t)STAGES * (RES ? 3 : 2) * N * threads * 16 : 0, sums = SPLIT ? 0 : sizeof(float) * (threads / a.lanes) * (size_t)a.dim;
    const size_t smem = ring > sums ? ring : sums;
    const auto kernel = rms_norm_grad_kernel<W, N, STAGES, SPLIT, RES, WT>;
    if (smem > 40960) CAST_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    return launch_chained(true, kernel, dim3(ctas), threads, smem, stream, 1, a);
}

template <int W, int N, int STAGES, bool SPLIT>
int launch_grad(const NormGradArgs& a, bool weight_fp32, unsigned ctas, cudaStream_t stream)
{
    if (a.dh) return weight_fp32 ? launch_grad<W, N, STAGES, SPLIT, true, float>(a, ctas, stream) : launch_grad<W, N, STAGES, SPLIT, true, uint16_t>(a, ctas, stream);
    return weight_fp32 ? launch_grad<W, N, STAGES, SPLIT, false, float>(a, ctas, stream) : launch_grad<W, N, STAGES, SPLIT, false, uint16_t>(a, ctas, stream);
}

int check_norm(const void* weight, int weight_fp32, int64_t tokens, int64_t dim, float eps)
{
    if (!weight) return CAST_ERR_NULL;
    if (tokens < 1 || tokens > 0x7FFFFFFF || dim < 1 || dim > kMostColumns) return CAST_ERR_SHAPE;
    if (!std::isfinite(eps) || eps < 0.0f) return CAST_ERR_HYPER;
    if ((uintptr_t)weight & (weight_fp32 ? 3u : 1u)) return CAST_ERR_ALIGN;
    return CAST_OK;
}

bool aligned(const void* p, unsigned bytes) { return ((uintptr_t)p & (bytes - 1u)) == 0; }

int norm_impl(const uint16_t* x, const uint16_t* residual, const void* weight, int weight_fp32, uint16_t* y, uint8_t* q, uint8_t* scales, uint16_t* h,
              int64_t tokens, int64_t dim, float eps, cudaStream_t stream)
{
    int rc;
    if (!x || (!y && (!q || !scales)) || (residual != nullptr) != (h != nullptr)) return CAST_ERR_NULL;
    if ((rc = check_norm(weight, weight_fp32, tokens, dim, eps)) != CAST_OK) return rc;
    if (!aligned(x, 2) || !aligned(residual, 2) || !aligned(y, 2) || !aligned(h, 2)) return CAST_ERR_ALIGN;
    const uint64_t n = (uint64_t)tokens * (uint64_t)dim;
    const void* const in[3] = {x, residual, weight};
    const uint64_t in_bytes[3] = {2 * n, 2 * n, (uint64_t)dim * (weight_fp32 ? 4u : 2u)};
    const void* const out[4] = {y, q, scales, h};
    const uint64_t out_bytes[4] = {2 * n, n, (uint64_t)tokens * (uint64_t)((dim + kGroup - 1) / kGroup), 2 * n};
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 3; ++i) {
            if (o == 3 && i < 2 && out[o] == in[i]) continue;          // the sum may take the place of one of its terms
            if (ranges_overlap(out[o], out_bytes[o], in[i], in_bytes[i])) return CAST_ERR_ALIAS;
        }
        for (int p = 0; p < o; ++p)
            if (ranges_overlap(out[o], out_bytes[o], out[p], out_bytes[p])) return CAST_ERR_ALIAS;
    }
    const void* ptrs[7] = {x, residual, weight, y, q, scales, h};
    if ((rc = check_device_memory(ptrs, 7)) != CAST_OK) return rc;
    const int w = dim % 8 == 0 && aligned(x, 16) && aligned(residual, 16) && aligned(weight, 16) && aligned(y, 16) && aligned(q, 8) && aligned(h, 16) ? 8 : 1;
    NormArgs a = {x, residual, weight, y, q, scales, h, (int32_t)tokens, (int32_t)dim, (int32_t)(dim / w), 0, eps};
    const Spread s = spread_of(a.units, w);
    a.lanes = s.lanes;
    const bool f = weight_fp32 != 0;
    if (w == 8) {
        if (!s.split) return s.n == 1 ? launch_norm<8, 1, false>(a, f, stream) : s.n == 2 ? launch_norm<8, 2, false>(a, f, stream) : launch_norm<8, 4, false>(a, f, stream);
        return s.n == 1 ? launch_norm<8, 1, true>(a, f, stream) : s.n == 2 ? launch_norm<8, 2, true>(a, f, stream) : launch_norm<8, 4, true>(a, f, stream);
    }
    if (!s.split) return launch_norm<1, 8, false>(a, f, stream);
    return s.n == 8 ? launch_norm<1, 8, true>(a, f, stream) : launch_norm<1, 32, true>(a, f, stream);
}

}  // namespace
}  // namespace cast

using namespace cast;

extern "C" int cast_rms_norm(const cast_bf16* x, const cast_bf16* residual, const void* weight, int weight_fp32, cast_bf16* y, cast_bf16* h,
                             int64_t tokens, int64_t dim, float eps, cast_stream_t stream)
{
    return norm_impl(x, residual, weight, weight_fp32, y, nullptr, nullptr, h, tokens, dim, eps, (cudaStream_t)stream);
}

extern "C" int cast_rms_norm_mx(const cast_bf16* x, const cast_bf16* residual, const void* weight, int weight_fp32, uint8_t* q, uint8_t* q_scales,
                                cast_bf16* h, int64_t tokens, int64_t dim, float eps, cast_stream_t stream)
{
    return norm_impl(x, residual, weight, weight_fp32, nullptr, q, q_scales, h, tokens, dim, eps, (cudaStream_t)stream);
}

extern "C" int cast_rms_norm_grad_workspace(int64_t tokens, int64_t dim, uint64_t* bytes)
{
    if (!bytes) return CAST_ERR_NULL;
    *bytes = 0;
    if (tokens < 1 || tokens > 0x7FFFFFFF || dim < 1 || dim > kMostColumns) return CAST_ERR_SHAPE;
    int sms = 0, rc;
    if ((rc = sm_count(&sms)) != CAST_OK) return rc;
    *bytes = grad_workspace(tokens, dim, sms);
    return CAST_OK;
}

extern "C" int cast_rms_norm_grad(const cast_bf16* grad_y, const cast_bf16* h, const void* weight, int weight_fp32, const cast_bf16* grad_h, cast_bf16* grad_x,
                                  float* grad_weight, int64_t tokens, int64_t dim, float eps, void* workspace, uint64_t workspace_bytes, cast_stream_t stream)
{
    int rc;
    if (!grad_y || !h || !grad_x || (grad_weight && !workspace)) return CAST_ERR_NULL;
    if ((rc = check_norm(weight, weight_fp32, tokens, dim, eps)) != CAST_OK) return rc;
    if (!aligned(grad_y, 2) || !aligned(h, 2) || !aligned(grad_h, 2) || !aligned(grad_x, 2) || !aligned(grad_weight, 4) || !aligned(workspace, 16)) return CAST_ERR_ALIGN;
    const uint64_t n = 2ull * (uint64_t)tokens * (uint64_t)dim;
    const void* const in[4] = {grad_y, h, grad_h, weight};
    const uint64_t in_bytes[4] = {n, n, n, (uint64_t)dim * (weight_fp32 ? 4u : 2u)};
    const void* const out[3] = {grad_x, grad_weight, grad_weight ? workspace : nullptr};
    const uint64_t out_bytes[3] = {n, 4ull * (uint64_t)dim, workspace_bytes};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 4; ++i) {
            if (o == 0 && i == 2 && out[o] == in[i]) continue;         // the gradient of the stream may be brought up to date in place
            if (ranges_overlap(out[o], out_bytes[o], in[i], in_bytes[i])) return CAST_ERR_ALIAS;
        }
        for (int p = 0; p < o; ++p)
            if (ranges_overlap(out[o], out_bytes[o], out[p], out_bytes[p])) return CAST_ERR_ALIAS;
    }
    int sms = 0;
    if ((rc = sm_count(&sms)) != CAST_OK) return rc;
    const int w = dim % 8 == 0 && aligned(grad_y, 16) && aligned(h, 16) && aligned(grad_h, 16) && aligned(grad_x, 16) && aligned(weight, 16) ? 8 : 1;
    NormGradArgs a = {grad_y, h, grad_h, weight, grad_x, grad_weight ? static_cast<float*>(workspace) : nullptr, (int32_t)tokens, (int32_t)dim,
                      (int32_t)(dim / w), 0, eps};
    const GradSpread g = grad_spread_of(a.units, w);
    const Spread& s = g.s;
    a.lanes = s.lanes;
    const unsigned ctas = (unsigned)grad_ctas(s, tokens, sms);
    if (grad_weight && workspace_bytes < grad_workspace(tokens, dim, sms)) return CAST_ERR_PLAN;
    const void* ptrs[7] = {grad_y, h, grad_h, weight, grad_x, grad_weight, grad_weight ? workspace : nullptr};
    if ((rc = check_device_memory(ptrs, 7)) != CAST_OK) return rc;
    const bool f = weight_fp32 != 0;
    const cudaStream_t st = (cudaStream_t)stream;
    if (w == 8) {
        if (!s.split)
            rc = s.n == 1 ? launch_grad<8, 1, 4, false>(a, f, ctas, st) : s.n == 2 ? launch_grad<8, 2, 4, false>(a, f, ctas, st) : launch_grad<8, 4, 2, false>(a, f, ctas, st);
        else if (s.n <= 2)
            rc = s.n == 1 ? launch_grad<8, 1, 4, true>(a, f, ctas, st) : launch_grad<8, 2, 4, true>(a, f, ctas, st);
        else
            rc = g.stages == 2 ? launch_grad<8, 4, 2, true>(a, f, ctas, st) : launch_grad<8, 4, 1, true>(a, f, ctas, st);
    } else {
        rc = !s.split ? launch_grad<1, 8, 1, false>(a, f, ctas, st) : s.n == 8 ? launch_grad<1, 8, 1, true>(a, f, ctas, st) : launch_grad<1, 32, 1, true>(a, f, ctas, st);
    }
    if (rc != CAST_OK || !grad_weight) return rc;
    return launch_chained(false, join_weight_grad_kernel, dim3((unsigned)((dim + 31) / 32)), 32 * kJoinWarps, 0, st, 1, (const float*)a.partial, grad_weight,
                          (int32_t)ctas, (int32_t)dim);
}
