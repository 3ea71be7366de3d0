// Root-mean-square norm of the rows of a residual stream, and its gradient.
//
//   forward    h = bf16(x + residual) (or h = x),  r = 1 / sqrt(mean(h^2) + eps),  y = weight h r
//   gradient   n = h r,  g = weight dy,  dx = r (g - n mean(g n)) + dh,  dweight = sum over the rows of dy n
//
// Forward: one pass; a row stays in registers between its sum of squares and its result.  `lanes` threads share a row, each with up to
// N accesses of W columns: 4 to 32 lanes of a warp (several rows per warp or CTA, no barrier), or a whole CTA.  Bounded by HBM: 16384 x 4096 with
// residual 79.5 us (537 MB, 6.75 TB/s), 4096 x 12288 61.6 us (6.54 TB/s); the 8-bit form of 8190 x 5120 52.6 us (295 MB, 5.6 TB/s) and 57 under
// the power limit: its instructions (two passes over a row in registers, groups' maxima, conversions) keep the issue slots busy.
//
// Gradient: the statistics of a row come from h again instead of being kept (one more multiply-add per column, 4 bytes per row less, nothing to
// pass on).  CTAs walk over rows with a stride; a thread owns the same columns of all of its rows and sums their part of
// dweight in registers.  The next rows are on their way to shared memory while one is worked on.  Each CTA leaves one fp32
// row of sums, and a second kernel adds those: no atomics, the same bits every time.  16384 x 4096 with the stream's gradient 83 us
// (537 MB, 6.5 TB/s), 86 to 88 under the power limit; 1000 x 768 5.7 us, two launches.
//
// Roundings: sums and statistics are fp32 (fp64 for rows whose squares leave the range of fp32), y and dx are rounded once; h is rounded to
// bf16 first, because that is the stream that is stored and normalised again by the backward pass.
#include <atomic>
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
    float inverse_dim;
    double inverse_dim64;     // 8-bit form
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

// A thread's sums of h^2 and of weight dy h over its columns of such a row, in fp64 and from memory again: rare, and
// outside of what the other rows' code keeps in registers.
template <int W>
__device__ __noinline__ double2 odd_sums(const uint16_t* h, const uint16_t* dy, const void* weight, bool weight_fp32, int dim, int lanes, int lane)
{
    double hh = 0.0, gh = 0.0;
    for (int c = lane * W; c < dim; c += lanes * W)
        for (int j = 0; j < W; ++j) {
            const double v = (double)bf16_low(h[c + j]);
            hh = fma(v, v, hh);
            const double w = (double)(weight_fp32 ? static_cast<const float*>(weight)[c + j] : bf16_low(static_cast<const uint16_t*>(weight)[c + j]));
            gh = fma((double)bf16_low(dy[c + j]) * w, v, gh);
        }
    return make_double2(hh, gh);
}

// A thread's sum of h^2 as a tree: an addition's operands have been through the same number of roundings, 2 + log2(N W / 4) of them at the end
// (squares of bf16 entries are exact in fp32).
template <int W, int N>
__device__ __forceinline__ float tree_of_squares(const typename Access<W>::Raw (&h)[N])
{
    constexpr int EIGHTS = (N * W + 7) / 8;
    float s[EIGHTS];
#pragma unroll
    for (int b = 0; b < EIGHTS; ++b) {
        float v[8], p[4];
        if constexpr (W == 8) {
            Access<8>::unpack(h[b], v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = bf16_low(h[b * 8 + j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = fmaf(v[2 * j], v[2 * j], v[2 * j + 1] * v[2 * j + 1]);
        s[b] = (p[0] + p[1]) + (p[2] + p[3]);
    }
    static_assert(EIGHTS <= 4, "two more additions at most");
    if constexpr (EIGHTS == 4) return (s[0] + s[1]) + (s[2] + s[3]);
    else if constexpr (EIGHTS == 3) return (s[0] + s[1]) + s[2];
    else if constexpr (EIGHTS == 2) return s[0] + s[1];
    else return s[0];
}

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

// Values in fp32 that lie this near to a border of the 8-bit form (units in the last place; two e4m3 values' middle, or a group's maximum at 448 times a
// power of two) are worked out again in fp64, so that values and scales are those of the exact norm.  With u = 2^-24, the most of a rounding, the mean square
// is off by 6 u where a row has a CTA (5 of a thread's sum, fp64 beyond, its own rounding) and by 12 u where it stays in a warp (5 more of the shuffles, one of
// 1/dim).  Its root's reciprocal has half of that and u, two products add 2 u: 6 or 9 u of a value, which are 6 m / 2 or 9 m / 2 units at a mantissa m.
// The borders' mantissas are 31/16 and 7/4 at most: less than 6 or 9 units, and borders are whole units away.
// (8190 x 5120: 52.6 us; a warp's sums in fp64, too, and 5 units there: 65536 x 256 19.9 instead of 18.8; fp32 throughout and 11 units: 53.6 and 18.8.
// Exact sums and the look for such values take 5 of the 52.6; one row in twenty is worked out again.)
template <bool SPLIT> constexpr uint32_t kNear = SPLIT ? 5 : 8;
// the last 20 bits as the upper ones, from kNear below their middle on: one multiply-add; the smaller, the nearer
__device__ __forceinline__ uint32_t distance_key(float scaled, uint32_t near) { return __float_as_uint(scaled) * 4096u + ((near - 0x80000u) << 12); }
// of a group's maximum to 1.75 times a power of two
__device__ __forceinline__ uint32_t scale_distance(uint32_t top, uint32_t near) { return (top & 0x7FFFFFu) + (near - 0x600000u); }

// 1 / sqrt(mean(h^2) + eps) of a row from memory in fp64, by `width` lanes of a warp; the row has been stored and the lanes synchronised.
template <int W>
__device__ __forceinline__ double exact_factor(const uint16_t* h, int dim, float eps, int width)
{
    double s = 0.0;
    for (int c = ((int)threadIdx.x & (width - 1)) * W; c < dim; c += width * W) {
        float v[W];
        Access<W>::unpack(*reinterpret_cast<const typename Access<W>::Raw*>(h + c), v);
#pragma unroll
        for (int j = 0; j < W; ++j) s = fma((double)v[j], (double)v[j], s);
    }
    for (int d = width >> 1; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    return 1.0 / sqrt(s / (double)dim + (double)eps);
}

// fp64 to fp32 such that a later rounding to fewer bits is that of the fp64 value: cut, with the last bit set where something was cut off.
__device__ __forceinline__ float to_odd(double v)
{
    const float f = __double2float_rz(v);
    return (double)f == v ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// The 8-bit values (x, y) and the scale (z) of one access in fp64.  A whole warp; everything by value, so that its other paths keep their registers.
template <int W, class WT>
__device__ __forceinline__ uint4 exact_group(typename Access<W>::Raw raw, const WT* weight, double r, bool in)
{
    float h[W], w[W];
    Access<W>::unpack(raw, h);
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = 0.0f;
    if (in) Access<W>::weights(weight, w);
    double y[W], top = 0.0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        y[j] = (double)h[j] * (double)w[j] * r;
        top = fmax(top, fabs(y[j]));
    }
#pragma unroll
    for (int d = kGroup / W / 2; d > 0; d >>= 1) top = fmax(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const uint32_t scale = group_scale(__float_as_uint(__double2float_ru(top)));
    const double inv = (double)inverse_scale(scale);
    if constexpr (W == 8) {
        return make_uint4(e4m3_pair(to_odd(y[0] * inv), to_odd(y[1] * inv)) | e4m3_pair(to_odd(y[2] * inv), to_odd(y[3] * inv)) << 16,
                          e4m3_pair(to_odd(y[4] * inv), to_odd(y[5] * inv)) | e4m3_pair(to_odd(y[6] * inv), to_odd(y[7] * inv)) << 16, scale, 0u);
    } else {
        return make_uint4(e4m3_pair(to_odd(y[0] * inv), 0.0f), 0u, scale, 0u);
    }
}

// The largest of three magnitudes as bits, NaN where one is.
__device__ __forceinline__ uint32_t largest(uint32_t top, float a, float b)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(__uint_as_float(top)), "f"(a), "f"(b));
    return __float_as_uint(r) & 0x7FFFFFFFu;
}

template <int W, int N, bool SPLIT, bool RES, bool MX, class WT>
__global__ void __launch_bounds__(SPLIT ? 1024 : 256)
rms_norm_kernel(const __grid_constant__ NormArgs a)
{
    using A = Access<W>;
    using Raw = typename A::Raw;
    __shared__ float part[kMostWarps];
    __shared__ double part64[MX ? 2 : 1][kMostWarps];
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
    float mean;
    if constexpr (MX) {
        const float square = tree_of_squares<W, N>(h);
        if constexpr (SPLIT) mean = (float)fma(row_sum<SPLIT>((double)square, a.lanes, part64[1]), a.inverse_dim64, (double)a.eps);
        else mean = fmaf(row_sum<SPLIT>(square, a.lanes, part), a.inverse_dim, a.eps);
    } else {
        float square = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[W];
            A::unpack(h[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) square = fmaf(v[j], v[j], square);
        }
        mean = fmaf(row_sum<SPLIT>(square, a.lanes, part), a.inverse_dim, a.eps);
    }
    float r = __frsqrt_rn(mean), pre = 1.0f;
    const bool odd = odd_row(mean);
    if (SPLIT ? odd : __any_sync(0xFFFFFFFFu, odd)) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[W];
            A::unpack(h[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) s = fma((double)v[j], (double)v[j], s);
        }
        s = row_sum<SPLIT>(s, a.lanes, part64[0]) / (double)a.dim + (double)a.eps;
        if (odd) {
            pre = odd_factor(s);
            r = (float)(1.0 / sqrt(s) / (double)pre);
        }
    }
    auto store_8_bits = [&](int c, const uint2& q, uint32_t scale) {
        if constexpr (W == 8) *reinterpret_cast<uint2*>(a.q + base + (int64_t)c * W) = q;
        else a.q[base + c] = (uint8_t)q.x;
        if (c % (kGroup / W) == 0) a.scales[row * ((a.dim + kGroup - 1) / kGroup) + c / (kGroup / W)] = (uint8_t)scale;
    };
    uint32_t nearest = 0xFFFFFFFFu, nearest_scale = 0xFFFFFFFFu, not_finite = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = i * a.lanes + lane;
        const bool in = active && c < a.units;
        float v[W], w[W];
        A::unpack(h[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = 0.0f;
        if (in) A::weights(static_cast<const WT*>(a.weight) + c * W, w);
        if (odd) {
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] *= pre;
        }
        // two bf16 entries multiply exactly: one rounding less than the other way round
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = v[j] * w[j] * r;
        if constexpr (!MX) {
            if (in) *reinterpret_cast<Raw*>(a.y + base + (int64_t)c * W) = A::pack(v);
        } else {
            // a group is 4 neighbouring lanes of 8 columns, or a warp of one column each; magnitudes are compared as bits, so that NaN counts
            // as the largest
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < W; j += 2) top = W == 1 ? __float_as_uint(v[0]) & 0x7FFFFFFFu : largest(top, v[j], v[(j + 1) % W]);
            if (!in) top = 0;
#pragma unroll
            for (int d = kGroup / W / 2; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            const uint32_t s = group_scale(top);
            const float inv = inverse_scale(s);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                v[j] *= inv;
                nearest = min(nearest, distance_key(v[j], kNear<SPLIT>));
            }
            nearest_scale = min(nearest_scale, scale_distance(top, kNear<SPLIT>));
            not_finite |= (s == 255u ? 1u : 0u) << i;
            if (!in) continue;
            if constexpr (W == 8) store_8_bits(c, make_uint2(e4m3_pair(v[0], v[1]) | e4m3_pair(v[2], v[3]) << 16, e4m3_pair(v[4], v[5]) | e4m3_pair(v[6], v[7]) << 16), s);
            else store_8_bits(c, make_uint2(e4m3_pair(v[0], 0.0f), 0u), s);
        }
    }
    if constexpr (MX) {
        if (__any_sync(0xFFFFFFFFu, nearest < (2 * kNear<SPLIT> + 1) << 12 || nearest_scale <= 2 * kNear<SPLIT>)) {
            __syncwarp();                            // the row's entries that other lanes stored; other warps' lie before the sum's barrier
            const uint16_t* stored = (RES ? a.h : a.x) + base;
            const double factor = exact_factor<W>(stored, active ? a.dim : 0, a.eps, SPLIT ? 32 : a.lanes);
#pragma unroll 1
            for (int i = 0; i < N; ++i) {
                const int c = i * a.lanes + lane;
                const bool in = active && c < a.units;
                Raw raw = A::zero();
                if (in) raw = *reinterpret_cast<const Raw*>(stored + c * W);
                const uint4 exact = exact_group<W, WT>(raw, static_cast<const WT*>(a.weight) + c * W, factor, in);
                if (in && !(not_finite >> i & 1u)) store_8_bits(c, make_uint2(exact.x, exact.y), exact.z);
            }
        }
    }
}

// The same for rows that begin anywhere (a width that is no multiple of 8), as long as all arrays lie alike: accesses are the aligned 16-byte blocks
// that a row touches, of which the first and the last belong to its neighbours in part.  Those are read whole where they lie inside the array and
// written by single columns.
template <int N, bool SPLIT, bool RES, class WT>
__global__ void __launch_bounds__(SPLIT ? 1024 : 256)
rms_norm_shifted_kernel(const __grid_constant__ NormArgs a)
{
    using A = Access<8>;
    __shared__ float part[kMostWarps];
    __shared__ double part64[kMostWarps];
    const int lane = SPLIT ? (int)threadIdx.x : (int)threadIdx.x & (a.lanes - 1);
    const int64_t row = SPLIT ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / a.lanes) + threadIdx.x / a.lanes;
    const bool active = SPLIT || row < a.tokens;
    const int64_t base = active ? row * a.dim : 0, all = (int64_t)a.tokens * a.dim;
    const int skip = (int)((uintptr_t)(a.x + base) & 15u) / 2, blocks = active ? (skip + a.dim + 7) / 8 : 0;
    const int64_t start = base - skip;               // entry of the array at which the row's first block begins, up to 7 before it
    auto load = [&](const uint16_t* p, int c) {
        const int64_t at = start + 8 * c;
        uint4 r = make_uint4(0u, 0u, 0u, 0u);
        if (at >= 0 && at + 8 <= all) {
            r = *reinterpret_cast<const uint4*>(p + at);
        } else {
            uint32_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = at + j >= 0 && at + j < all ? p[at + j] : 0u;
            r = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
        return r;
    };
    auto store = [&](uint16_t* p, int c, const uint4& r) {
        uint16_t* q = p + start + 8 * c;
        const int col = 8 * c - skip;
        if (col >= 0 && col + 8 <= a.dim) {
            *reinterpret_cast<uint4*>(q) = r;
        } else {
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j >= 0 && col + j < a.dim) q[j] = (uint16_t)(j % 2 ? w[j / 2] >> 16 : w[j / 2]);
        }
    };
    // an entry of the neighbours counts as 0
    auto mask = [&](int c, float (&v)[8]) {
        const int col = 8 * c - skip;
        if (col >= 0 && col + 8 <= a.dim) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < 0 || col + j >= a.dim) v[j] = 0.0f;
    };
    uint4 h[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = i * a.lanes + lane;
        h[i] = make_uint4(0u, 0u, 0u, 0u);
        if (c < blocks) h[i] = load(a.x, c);
    }
    if constexpr (RES) {
        uint4 r[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            r[i] = make_uint4(0u, 0u, 0u, 0u);
            if (c < blocks) r[i] = load(a.residual, c);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * a.lanes + lane;
            float u[8], v[8];
            A::unpack(h[i], u);
            A::unpack(r[i], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] += v[j];
            h[i] = A::pack(u);
            if (c < blocks) store(a.h, c, h[i]);
        }
    }
    float square = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[8];
        A::unpack(h[i], v);
        mask(i * a.lanes + lane, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) square = fmaf(v[j], v[j], square);
    }
    const float mean = fmaf(row_sum<SPLIT>(square, a.lanes, part), a.inverse_dim, a.eps);
    float r = __frsqrt_rn(mean), pre = 1.0f;
    const bool odd = odd_row(mean);
    if (SPLIT ? odd : __any_sync(0xFFFFFFFFu, odd)) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[8];
            A::unpack(h[i], v);
            mask(i * a.lanes + lane, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s = fma((double)v[j], (double)v[j], s);
        }
        s = row_sum<SPLIT>(s, a.lanes, part64) / (double)a.dim + (double)a.eps;
        if (odd) {
            pre = odd_factor(s);
            r = (float)(1.0 / sqrt(s) / (double)pre);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = i * a.lanes + lane, col = 8 * c - skip;
        if (c >= blocks) continue;
        float v[8], w[8];
        A::unpack(h[i], v);
        const WT* weight = static_cast<const WT*>(a.weight) + col;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float one[1] = {0.0f};
            if (col + j >= 0 && col + j < a.dim) Access<1>::weights(weight + j, one);
            w[j] = one[0];
        }
        if (odd) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= pre;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] * w[j] * r;
        store(a.y, c, A::pack(v));
    }
}

// How a row is spread: lanes and accesses per lane (N, one of the instantiated ones); lanes <= 32 are lanes of one warp.
struct Spread {
    int lanes, n;
    bool split;
};

Spread spread_of(int64_t units, int w, bool res, bool mx)
{
    if (w == 8) {
        if (units <= 128) {                   // up to 1024 columns: in a warp
            int lanes = 4;                    // two accesses or more each: 65536 x 128 6.65 us, with one each 8.5
            while (lanes < 32 && 2 * lanes < units) lanes *= 2;
            return {lanes, (int)((units + lanes - 1) / lanes), false};
        }
        // Fewer accesses per thread leave SMs with too few bytes in flight behind the barrier of a row, more of them with too few CTAs (us;
        // 16384 x 4096 with residual: one 84.7, two 79.8, four 80.6; to 8 bits: two 87.6, four 83.4; without residual, 8192 x 4096: one 34.6, two 27.6,
        // three 25.5, four 22.9; 4096 x 12288 with residual: two 80, four 61.7, eight 69).
        const bool plain = res && !mx;
        const int n = units <= 256 ? (plain ? 1 : 2) : !plain ? 4 : units <= 512 ? 2 : units <= 768 ? 3 : 4;
        return {(int)((units + n * 32 - 1) / (n * 32)) * 32, n, true};
    }
    // single columns: 32 of them spill up to 576 bytes at the 64 registers of 1024 threads; rows beyond 8192 columns take them only off the 16-byte grid
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

// One and three accesses per thread of a CTA are taken with a residual and a bf16 result only.
template <int N>
int launch_plain_norm(const NormArgs& a, bool weight_fp32, cudaStream_t stream)
{
    return weight_fp32 ? launch_norm<8, N, true, true, false, float>(a, stream) : launch_norm<8, N, true, true, false, uint16_t>(a, stream);
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

template <int N, bool SPLIT>
int launch_shifted(const NormArgs& a, bool weight_fp32, cudaStream_t stream)
{
    const unsigned threads = SPLIT ? (unsigned)a.lanes : 256u, rows = SPLIT ? 1u : threads / (unsigned)a.lanes, grid = ((unsigned)a.tokens + rows - 1) / rows;
    if (a.residual && weight_fp32) rms_norm_shifted_kernel<N, SPLIT, true, float><<<grid, threads, 0, stream>>>(a);
    else if (a.residual) rms_norm_shifted_kernel<N, SPLIT, true, uint16_t><<<grid, threads, 0, stream>>>(a);
    else if (weight_fp32) rms_norm_shifted_kernel<N, SPLIT, false, float><<<grid, threads, 0, stream>>>(a);
    else rms_norm_shifted_kernel<N, SPLIT, false, uint16_t><<<grid, threads, 0, stream>>>(a);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    return CAST_OK;
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
    int32_t window;           // W == 1: entries of shared memory for a row of one array
    float eps;
    float inverse_dim;
};

__device__ __forceinline__ void copy_async(uint32_t shared, const void* global, int bytes)      // 16 bytes, those beyond `bytes` as zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(shared), "l"(global), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(PENDING) : "memory"); }

// A thread's N parts of a row: with W == 8 the 4 pairs of neighbouring columns of an access, with W == 1 one pair of columns `lanes` apart.
template <int W>
struct Part {
    static constexpr int kPairs = W == 8 ? 4 : 1;
    static __device__ __forceinline__ int column(int i, int e, int lanes, int lane) { return W == 8 ? (i * lanes + lane) * 8 + e : (2 * i + e) * lanes + lane; }
};

// STAGES rows of the arrays on their way through shared memory.  W == 8: every thread copies the accesses that it will read itself,
// [STAGES][arrays][N][threads], so that no barrier is needed.  W == 1: the threads of a row copy the 16-byte blocks that the row
// touches (rows begin anywhere), and read single columns of one another's blocks behind a barrier.
template <int W, int N, int STAGES, bool RES>
struct Ring {
    static constexpr int kArrays = RES ? 3 : 2;
    const NormGradArgs& a;
    int lane, sub, rows;
    uint32_t slot;                                   // shared address of this thread's first access (W == 8), or of the ring
    uint32_t apart;                                  // W == 8: bytes between a thread's slots
    int64_t row, step;                               // the next row to fetch
    const uint16_t* next[kArrays];                   // W == 8: its entries
    int first[W == 8 ? 1 : kArrays];                 // W == 1: where the current row begins

    __device__ __forceinline__ const uint16_t* source(int k) const { return k == 0 ? a.h : k == 1 ? a.dy : a.dh; }
    __device__ __forceinline__ Ring(const NormGradArgs& args, const uint4* shared, int lane_, int sub_, int rows_, int64_t row_, int64_t step_)
        : a(args), lane(lane_), sub(sub_), rows(rows_), slot(shared_address(shared) + (W == 8 ? threadIdx.x * 16u : 0u)), apart(blockDim.x * 16u), row(row_), step(step_)
    {
#pragma unroll
        for (int k = 0; k < kArrays; ++k) next[k] = source(k) + row * a.dim;
    }
    // The next row, into `stage`.
    __device__ __forceinline__ void fetch(int stage)
    {
        if (row < a.tokens) {
#pragma unroll
            for (int k = 0; k < kArrays; ++k) {
                if constexpr (W == 8) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int c = i * a.lanes + lane;
                        copy_async(slot + ((stage * kArrays + k) * N + i) * apart, next[k] + (c < a.units ? c * 8 : 0), c < a.units ? 16 : 0);
                    }
                } else {
                    const uint16_t *begin = source(k), *end = begin + (int64_t)a.tokens * a.dim, *from = next[k];
                    const int skip = (int)((uintptr_t)from & 15u) / 2, blocks = (skip + a.dim + 7) / 8;
                    const uint32_t to = slot + ((stage * kArrays + k) * rows + sub) * a.window * 2;
                    for (int c = lane; c < blocks; c += a.lanes) {
                        const uint16_t* p = from - skip + 8 * c;
                        if (p >= begin) {
                            copy_async(to + 16 * c, p, (int)min((int64_t)16, (int64_t)(end - p) * 2));
                        } else {
                            // the array begins inside a block
                            for (int j = (int)(begin - p); j < 8 && p + j < end; ++j) asm volatile("st.shared.u16 [%0], %1;" :: "r"(to + 16 * c + 2 * j), "h"(p[j]) : "memory");
                        }
                    }
                }
            }
        }
        copies_commit();
        row += step;
#pragma unroll
        for (int k = 0; k < kArrays; ++k) next[k] += step * a.dim;
    }
    // W == 1: the row at hand
    __device__ __forceinline__ void turn_to(int64_t at, int stage)
    {
        if constexpr (W == 1) {
#pragma unroll
            for (int k = 0; k < kArrays; ++k)
                first[k] = ((stage * kArrays + k) * rows + sub) * a.window + (int)((uintptr_t)(source(k) + at * a.dim) & 15u) / 2;
        }
    }
    __device__ __forceinline__ uint16_t entry(int at) const
    {
        uint16_t v;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(slot + at * 2) : "memory");
        return v;
    }
    __device__ __forceinline__ void get(int k, int i, int stage, float2 (&v)[Part<W>::kPairs]) const
    {
        if constexpr (W == 8) {
            uint4 r;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(slot + ((stage * kArrays + k) * N + i) * apart) : "memory");
            Pairs::unpack(r, v);
        } else {
            const int c = Part<1>::column(i, 0, a.lanes, lane), d = Part<1>::column(i, 1, a.lanes, lane);
            v[0] = make_float2(c < a.dim ? bf16_low(entry(first[k] + c)) : 0.0f, d < a.dim ? bf16_low(entry(first[k] + d)) : 0.0f);
        }
    }
};

// Rows of 776 to 4096 columns: three on their way, two CTAs of up to 256 threads per SM with 128 registers, so that a row stays in
// registers between its two halves.  (16384 x 4096 in us, in short runs and under the power limit, where instructions count: 83.0 / 86.0 to 88;
// read from shared memory twice, 80 registers: 81.6 / 94.6; two rows and four CTAs with 64 registers: 87.0 / 96.1; four rows, two CTAs: 91.2 / 96.5.)
template <int W, int N, int STAGES, bool SPLIT> constexpr bool kMiddleRow = SPLIT && W == 8 && N == 2 && STAGES == 3;
// Threads that a CTA has at most, and CTAs that the registers are to hold.
template <int W, int N, int STAGES, bool SPLIT> constexpr int grad_threads()
{
    return !SPLIT || kMiddleRow<W, N, STAGES, SPLIT> ? 256 : N * Part<W>::kPairs <= 8 || (W == 8 && STAGES == 2) ? 512 : 1024;
}
template <int W, int N, int STAGES, bool SPLIT> constexpr int grad_blocks() { return !SPLIT || (W == 8 && N == 2) ? 2 : 1; }

template <int W, int N, int STAGES, bool SPLIT, bool RES, class WT>
__global__ void __launch_bounds__(grad_threads<W, N, STAGES, SPLIT>(), grad_blocks<W, N, STAGES, SPLIT>())
rms_norm_grad_kernel(const __grid_constant__ NormGradArgs a)
{
    constexpr int Q = Part<W>::kPairs;
    extern __shared__ uint4 dynamic[];               // the ring; !SPLIT, afterwards: [rows of the CTA][dim] sums
    __shared__ __align__(16) float2 part[2][kMostWarps];
    __shared__ double part64[2][kMostWarps];
    if (SPLIT && threadIdx.x < 2) part[threadIdx.x][(blockDim.x >> 5) & 31] = both(0.0f);       // behind an odd number of warps; set before the first barrier
    const int lane = SPLIT ? (int)threadIdx.x : (int)threadIdx.x & (a.lanes - 1);
    const int rows = SPLIT ? 1 : (int)blockDim.x / a.lanes, sub = SPLIT ? 0 : (int)threadIdx.x / a.lanes;
    float2 dw[N][Q];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < Q; ++j) dw[i][j] = both(0.0f);
    auto weight = [&](int i, float2 (&w)[Q]) {
        const WT* p = static_cast<const WT*>(a.weight);
        const int c = Part<W>::column(i, 0, a.lanes, lane);
#pragma unroll
        for (int j = 0; j < Q; ++j) w[j] = both(0.0f);
        if constexpr (W == 8) {
            if (c < a.dim) Pairs::weights(p + c, w);
        } else {
            const int d = Part<W>::column(i, 1, a.lanes, lane);
            float v[1];
            if (c < a.dim) { Access<1>::weights(p + c, v); w[0].x = v[0]; }
            if (d < a.dim) { Access<1>::weights(p + d, v); w[0].y = v[0]; }
        }
    };
    // a row stays in registers between its two halves, or is read from shared memory twice
    constexpr bool KEPT = N * Q <= 8 && (!SPLIT || W == 1 || kMiddleRow<W, N, STAGES, SPLIT>);
    // where an odd row's factor enters, by what the others' code pays for it: with g and m, or with what becomes of them (8192 x 5120: 77 and 55.5 us;
    // 4096 x 2560: 16.4 and 16.6)
    constexpr bool EARLY = KEPT && W == 8;
    constexpr bool WEIGHTS = N * Q <= 12;            // and the weights of a thread's columns for good
    float2 kept[WEIGHTS ? N : 1][Q];
    if constexpr (WEIGHTS) {
#pragma unroll
        for (int i = 0; i < N; ++i) weight(i, kept[i]);
    }
    const int64_t step = (int64_t)gridDim.x * rows;
    int64_t row0 = (int64_t)blockIdx.x * rows;
    Ring<W, N, STAGES, RES> ring(a, dynamic, lane, sub, rows, row0 + sub, step);
#pragma unroll
    for (int k = 0; k + 1 < STAGES; ++k) ring.fetch(k);
    int stage = 0;
    for (int turn = 0; row0 < a.tokens; row0 += step, turn ^= 1, stage = stage + 1 == STAGES ? 0 : stage + 1) {
        const int64_t row = row0 + sub;
        const int free = stage == 0 ? STAGES - 1 : stage - 1;         // the row before was there
        if constexpr (W == 8) {
            ring.fetch(free);
            copies_wait<STAGES - 1>();
        } else if constexpr (STAGES > 1) {
            copies_wait<STAGES - 2>();
            if constexpr (SPLIT) __syncthreads(); else __syncwarp();   // everyone's blocks are there, and the row before has been read
            ring.fetch(free);
        } else {
            if constexpr (SPLIT) __syncthreads(); else __syncwarp();
            ring.fetch(free);
            copies_wait<0>();
            if constexpr (SPLIT) __syncthreads(); else __syncwarp();
        }
        const bool active = row < a.tokens;
        ring.turn_to(active ? row : 0, stage);
        float2 u[KEPT ? N : 1][Q], g[KEPT ? N : 1][Q], v[KEPT ? N : 1][Q];
        float2 hh = both(0.0f), gh = both(0.0f);     // sums of h^2 and of g h
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = KEPT ? i : 0;
            ring.get(0, i, stage, u[e]);
            ring.get(1, i, stage, v[e]);
            if (W == 1 && !active) u[e][0] = v[e][0] = both(0.0f);
            float2 w[Q];
            if constexpr (!WEIGHTS) weight(i, w);
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                g[e][j] = mul2(v[e][j], WEIGHTS ? kept[WEIGHTS ? i : 0][j] : w[j]);
                hh = fma2(u[e][j], u[e][j], hh);
                gh = fma2(g[e][j], u[e][j], gh);
            }
        }
        float2 s = make_float2(hh.x + hh.y, gh.x + gh.y);
        for (int d = (SPLIT ? 32 : a.lanes) >> 1; d > 0; d >>= 1)
            s = add2(s, make_float2(__shfl_xor_sync(0xFFFFFFFFu, s.x, d), __shfl_xor_sync(0xFFFFFFFFu, s.y, d)));
        if constexpr (SPLIT) {
            // two buffers: a warp may be one row ahead of another, not two
            if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = s;
            __syncthreads();
            // two warps' sums by one load; where their number is odd the last one is 0
            s = both(0.0f);
            for (int i = 0; i < (int)(blockDim.x >> 5); i += 2) {
                const float4 two = *reinterpret_cast<const float4*>(&part[turn][i]);
                s = add2(s, add2(make_float2(two.x, two.y), make_float2(two.z, two.w)));
            }
        }
        const float mean = fmaf(s.x, a.inverse_dim, a.eps);
        float r = __frsqrt_rn(mean), scaled = r;                        // n = h * scaled
        float m = s.y * a.inverse_dim * r;                              // mean(g n)
        float pre = 1.0f;
        const bool odd = odd_row(mean) || !(fabsf(s.y) < 0x1p100f);     // or a sum of products that may have left the range
        if (SPLIT ? odd : __any_sync(0xFFFFFFFFu, odd)) {
            const double2 own = odd_sums<W>(a.h + row * a.dim, a.dy + row * a.dim, a.weight, std::is_same<WT, float>::value, active ? a.dim : 0, a.lanes, lane);
            if constexpr (SPLIT) __syncthreads();                        // the row before may have been an odd one, too
            const double s64 = row_sum<SPLIT>(own.x, a.lanes, part64[0]) / (double)a.dim + (double)a.eps;
            const double m64 = row_sum<SPLIT>(own.y, a.lanes, part64[1]) / (double)a.dim;
            if (odd) {
                const double r64 = 1.0 / sqrt(s64);
                if (odd_row(mean)) pre = odd_factor(s64);
                scaled = (float)(r64 / (double)pre);
                r = pre;                                                // 1/sqrt(mean) itself may have left the range: d times scaled, then pre
                m = (float)(EARLY ? m64 * r64 * (double)scaled : m64 * r64);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = Part<W>::column(i, 0, a.lanes, lane), e = KEPT ? i : 0;
            if (!active || c >= a.dim) continue;
            if constexpr (!KEPT) {
                float2 w[Q];
                ring.get(0, i, stage, u[0]);
                ring.get(1, i, stage, v[0]);
                if constexpr (!WEIGHTS) weight(i, w);
#pragma unroll
                for (int j = 0; j < Q; ++j) g[0][j] = mul2(v[0][j], WEIGHTS ? kept[WEIGHTS ? i : 0][j] : w[j]);
            }
            if (odd) {
#pragma unroll
                for (int j = 0; j < Q; ++j) {
                    u[e][j] = mul2(u[e][j], both(pre));
                    if (EARLY) g[e][j] = mul2(g[e][j], both(scaled));
                }
            }
            float2 o[Q];
            if constexpr (RES) ring.get(2, i, stage, o);
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                const float2 n = mul2(u[e][j], both(scaled));
                dw[i][j] = fma2(v[e][j], n, dw[i][j]);
                float2 d = fma2(n, both(-m), g[e][j]);
                if (!EARLY && odd) d = mul2(d, both(scaled));
                o[j] = RES ? fma2(both(r), d, o[j]) : mul2(both(r), d);
            }
            uint16_t* to = a.dx + row * a.dim + c;
            if constexpr (W == 8) {
                *reinterpret_cast<uint4*>(to) = Pairs::pack(o);
            } else {
                const uint32_t two = bf16_pair(o[0].x, o[0].y);
                to[0] = (uint16_t)two;
                if (c + a.lanes < a.dim) to[a.lanes] = (uint16_t)(two >> 16);
            }
        }
    }
    chain_next();
    copies_wait<0>();
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.x * a.dim;
    float* sums = reinterpret_cast<float*>(dynamic);
    if constexpr (!SPLIT) __syncthreads();           // the ring has been read
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = Part<W>::column(i, 0, a.lanes, lane);
        if (c >= a.dim) continue;
        float* to = (SPLIT ? out : sums + sub * a.dim) + c;
        if constexpr (W == 8) {
            reinterpret_cast<float4*>(to)[0] = make_float4(dw[i][0].x, dw[i][0].y, dw[i][1].x, dw[i][1].y);
            reinterpret_cast<float4*>(to)[1] = make_float4(dw[i][2].x, dw[i][2].y, dw[i][3].x, dw[i][3].y);
        } else {
            to[0] = dw[i][0].x;
            if (c + a.lanes < a.dim) to[a.lanes] = dw[i][0].y;
        }
    }
    if constexpr (!SPLIT) {
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

// Entries that a row of `dim` columns takes in shared memory when it begins anywhere.
int64_t window_of(int64_t dim) { return (dim + 7 + 7) / 8 * 8; }

constexpr int kMostRingBytes = 220000;       // of an SM's 227 KB: the kernel's static shared memory and what the system takes of every CTA beside it

struct GradSpread {
    int lanes, n;
    bool split;
    int stages;
    int64_t bytes;            // of shared memory
    int held;                 // CTAs that an SM holds
};

GradSpread grad_spread_of(int64_t dim, int w, bool res)
{
    GradSpread g = {};
    const int64_t units = dim / w, arrays = res ? 3 : 2;
    if (w == 8) {
        if (units <= 96) {                    // up to 768 columns: in a warp (65536 x 1024: in a warp 98 us, in two 92; x 640: 20.5, 24.6 for 16384)
            g.lanes = 8;
            while (g.lanes < 32 && g.lanes < units) g.lanes *= 2;
            g.n = (int)((units + g.lanes - 1) / g.lanes);
            g.stages = g.n <= 2 ? 4 : 2;
        } else {
            g.split = true;
            g.n = units <= 1024 ? 2 : 4;
            g.lanes = (int)((units + g.n * 32 - 1) / (g.n * 32)) * 32;
            g.stages = units <= 512 ? 3 : units <= 2048 ? 2 : 1;
        }
        g.bytes = g.stages * arrays * g.n * (g.split ? g.lanes : 256) * 16;
    } else {
        g.split = dim > 256;
        g.n = !g.split ? 4 : dim <= 8192 ? 8 : 16;
        g.lanes = !g.split ? 32 : (int)((dim + g.n * 64 - 1) / (g.n * 64)) * 32;
        const int64_t row = arrays * window_of(dim) * 2 * (g.split ? 1 : 256 / g.lanes);
        g.stages = g.n <= 8 ? (4 * row <= kMostRingBytes / 2 ? 4 : 2) : 2 * row <= kMostRingBytes ? 2 : 1;
        g.bytes = g.stages * row;
    }
    const int64_t sums = g.split ? 0 : 4 * dim * (256 / g.lanes);
    if (g.bytes < sums) g.bytes = sums;
    const int threads = g.split ? g.lanes : 256;
    g.held = (int)(kMostRingBytes / (g.bytes + 2048));
    const int by_registers = g.split && w == 8 && units > 512 && units <= 1024 ? 2 : threads <= 512 ? 512 / threads : 1;
    if (g.held > by_registers) g.held = by_registers;
    if (g.held < 1) g.held = 1;
    return g;
}

int sm_count(int* sms)
{
    int device = 0;
    CAST_CUDA_TRY(cudaGetDevice(&device));
    CAST_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
    return CAST_OK;
}

// CTAs of the gradient kernel: what the SMs hold at a time; fewer tokens than four rows for each of those, but more than fill two per SM, take
// fewer, since every one of them leaves a row of sums (1000 x 1024: 7.9 us with a CTA each, 6.0 with two per SM).
int64_t grad_ctas(const GradSpread& g, int64_t tokens, int sms)
{
    const int64_t rows = g.split ? 1 : 256 / g.lanes, groups = (tokens + rows - 1) / rows, held = (int64_t)sms * g.held;
    const int64_t quarter = groups / 4 > 2 * sms ? groups / 4 : 2 * sms, most = quarter < held ? quarter : held;
    return groups < most ? groups : most;
}

// Workspace for every form of the call: which one it takes depends on its pointers.
uint64_t grad_workspace(int64_t tokens, int64_t dim, int sms)
{
    int64_t most = 0;
    for (int w = 1; w <= 8; w += 7)
        for (int res = 0; res < 2; ++res) {
            const int64_t n = dim % w == 0 ? grad_ctas(grad_spread_of(dim, w, res != 0), tokens, sms) : 0;
            if (n > most) most = n;
        }
    return sizeof(float) * (uint64_t)most * (uint64_t)dim;
}

template <int W, int N, int STAGES, bool SPLIT, bool RES, class WT>
int launch_grad(const NormGradArgs& a, const GradSpread& g, unsigned ctas, cudaStream_t stream)
{
    const auto kernel = rms_norm_grad_kernel<W, N, STAGES, SPLIT, RES, WT>;
    // Once per kernel and device, and for every width at a time: the limit belongs to the kernel, so that a smaller one set by another thread would
    // refuse this one's launch.
    static std::atomic<uint64_t> allowed{0};
    int device = 0;
    CAST_CUDA_TRY(cudaGetDevice(&device));
    if (device >= 64 || !(allowed.load(std::memory_order_relaxed) >> device & 1u)) {
        CAST_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostRingBytes));
        if (device < 64) allowed.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    return launch_chained(true, kernel, dim3(ctas), SPLIT ? (unsigned)a.lanes : 256u, (size_t)g.bytes, stream, 1, a);
}

template <int W, int N, int STAGES, bool SPLIT>
int launch_grad(const NormGradArgs& a, const GradSpread& g, bool weight_fp32, unsigned ctas, cudaStream_t stream)
{
    if (a.dh) return weight_fp32 ? launch_grad<W, N, STAGES, SPLIT, true, float>(a, g, ctas, stream) : launch_grad<W, N, STAGES, SPLIT, true, uint16_t>(a, g, ctas, stream);
    return weight_fp32 ? launch_grad<W, N, STAGES, SPLIT, false, float>(a, g, ctas, stream) : launch_grad<W, N, STAGES, SPLIT, false, uint16_t>(a, g, ctas, stream);
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
    NormArgs a = {x, residual, weight, y, q, scales, h, (int32_t)tokens, (int32_t)dim, (int32_t)(dim / w), 0, eps, 1.0f / (float)dim, 1.0 / (double)dim};
    const Spread s = spread_of(a.units, w, residual != nullptr, q != nullptr);
    a.lanes = s.lanes;
    const bool f = weight_fp32 != 0;
    if (w == 8) {
        if (!s.split)
            return s.n == 1   ? launch_norm<8, 1, false>(a, f, stream)
                   : s.n == 2 ? launch_norm<8, 2, false>(a, f, stream)
                   : s.n == 3 ? launch_norm<8, 3, false>(a, f, stream)
                              : launch_norm<8, 4, false>(a, f, stream);
        return s.n == 1   ? launch_plain_norm<1>(a, f, stream)
               : s.n == 2 ? launch_norm<8, 2, true>(a, f, stream)
               : s.n == 3 ? launch_plain_norm<3>(a, f, stream)
                          : launch_norm<8, 4, true>(a, f, stream);
    }
    const uintptr_t place = (uintptr_t)x;
    const bool alike = !(((uintptr_t)residual ^ (residual ? place : 0)) & 15u) && !(((uintptr_t)h ^ (h ? place : 0)) & 15u) && !(((uintptr_t)y ^ place) & 15u);
    if (!q && alike && dim > 8) {
        // 16-byte accesses all the same: 4096 x 4097 with residual 30 us, by single columns 50
        const int64_t blocks = (dim + 14) / 8;       // of a row, at most
        if (blocks <= 128) {
            a.lanes = 4;
            while (a.lanes < 32 && 2 * a.lanes < blocks) a.lanes *= 2;
            return blocks <= 2 * a.lanes ? launch_shifted<2, false>(a, f, stream) : launch_shifted<4, false>(a, f, stream);
        }
        const int n = blocks <= 512 ? 2 : 4;
        a.lanes = (int32_t)((blocks + n * 32 - 1) / (n * 32)) * 32;
        if (a.lanes <= 1024) return n == 2 ? launch_shifted<2, true>(a, f, stream) : launch_shifted<4, true>(a, f, stream);
        a.lanes = s.lanes;
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
    const GradSpread g = grad_spread_of(dim, w, grad_h != nullptr);
    const NormGradArgs a = {grad_y, h, grad_h, weight, grad_x, grad_weight ? static_cast<float*>(workspace) : nullptr, (int32_t)tokens, (int32_t)dim,
                            (int32_t)(dim / w), g.lanes, (int32_t)window_of(dim), eps, 1.0f / (float)dim};
    const unsigned ctas = (unsigned)grad_ctas(g, tokens, sms);
    if (grad_weight && workspace_bytes < grad_workspace(tokens, dim, sms)) return CAST_ERR_PLAN;
    const void* ptrs[7] = {grad_y, h, grad_h, weight, grad_x, grad_weight, grad_weight ? workspace : nullptr};
    if ((rc = check_device_memory(ptrs, 7)) != CAST_OK) return rc;
    const bool f = weight_fp32 != 0;
    const cudaStream_t st = (cudaStream_t)stream;
    if (w == 8) {
        if (!g.split)
            rc = g.n == 1   ? launch_grad<8, 1, 4, false>(a, g, f, ctas, st)
                 : g.n == 2 ? launch_grad<8, 2, 4, false>(a, g, f, ctas, st)
                            : launch_grad<8, 3, 2, false>(a, g, f, ctas, st);
        else
            rc = g.n == 4 ? (g.stages == 2 ? launch_grad<8, 4, 2, true>(a, g, f, ctas, st) : launch_grad<8, 4, 1, true>(a, g, f, ctas, st))
                 : g.stages == 3 ? launch_grad<8, 2, 3, true>(a, g, f, ctas, st)
                                 : launch_grad<8, 2, 2, true>(a, g, f, ctas, st);
    } else if (!g.split) {
        rc = launch_grad<1, 4, 4, false>(a, g, f, ctas, st);
    } else if (g.n == 8) {
        rc = g.stages == 4 ? launch_grad<1, 8, 4, true>(a, g, f, ctas, st) : launch_grad<1, 8, 2, true>(a, g, f, ctas, st);
    } else {
        rc = g.stages == 2 ? launch_grad<1, 16, 2, true>(a, g, f, ctas, st) : launch_grad<1, 16, 1, true>(a, g, f, ctas, st);
    }
    if (rc != CAST_OK || !grad_weight) return rc;
    return launch_chained(false, join_weight_grad_kernel, dim3((unsigned)((dim + 31) / 32)), 32 * kJoinWarps, 0, st, 1, (const float*)a.partial, grad_weight,
                          (int32_t)ctas, (int32_t)dim);
}
