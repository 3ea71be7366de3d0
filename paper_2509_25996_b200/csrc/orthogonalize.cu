// Newton-Schulz orthogonalisation of updates (as the Muon optimiser applies it to hidden matrices):
//     X = U / (|U|_F + eps),   steps times  X <- a X + (b A + c A A) X,  A = X X^T,   out = scale X
// and X <- a X + X (b A + c A A) with A = X^T X where there are more rows than columns, so that A is the smaller square.
//
// Each step is three products on the tensor cores over all matrices of the call at once:
//     A = X X^T               symmetric: only tiles on and below the diagonal, each stored twice (once transposed)
//     P = b A + c A A         symmetric likewise; b A is added by the epilogue
//     X' = a X + P X          a X is added by the epilogue
// Operands are never transposed in memory: X is read K-major in one product and MN-major in the other.
//
// Numbers: the operands are fp16, not bf16.  Every value is bounded (|X| singular values stay near 1), so the range is
// enough and the 3 more bits of significand are worth 8 times less rounding noise.  X is held as hi + lo, two fp16 words scaled
// by 2^12 (22 bits): the products read hi, a X reads both.  That matters because a = 3.4 per step amplifies small singular
// directions 500-fold over five steps: noise from rounding X itself would be amplified with them, while noise that enters
// through the products is confined to directions that are large already.  A and P (b A + c A A, without a I) are plain fp16.
#include <algorithm>
#include <cmath>
#include <new>

#include <cuda_fp16.h>

#include "embed.cuh"
#include "tile_product.cuh"

namespace cast {
namespace {

using namespace product;

constexpr float kX = 4096.0f;               // X is stored times this
constexpr int kGroup = 64;                  // matrices per launch at most
constexpr int64_t kGroupElems = 64 << 20;   // ... and elements, which bounds the workspace
constexpr int kNormBlocks = 128;

struct PtrTable { const void* p[kGroup]; };
struct OutTable { uint16_t* p[kGroup]; };

__device__ __forceinline__ float f16_lo(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu))); }
__device__ __forceinline__ float f16_hi(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
// round to nearest, and to the largest finite value beyond the range (coefficients under which X grows without bound)
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_b16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ------------------------------------------------------------------------------------------------ norm and first X

template <bool BF16, int VEC>
__device__ __forceinline__ void load_update(const void* u, int64_t unit, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        if constexpr (BF16) v[0] = __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(u) + unit) << 16);
        else v[0] = __ldg(static_cast<const float*>(u) + unit);
    } else if constexpr (BF16) {
        const uint4 x = __ldg(static_cast<const uint4*>(u) + unit);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    } else {
        const float4 x = __ldg(static_cast<const float4*>(u) + 2 * unit), y = __ldg(static_cast<const float4*>(u) + 2 * unit + 1);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
}

__device__ __forceinline__ double block_sum(double x)
{
    __shared__ double part[8];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    for (int i = 0; i < 8; ++i) x += part[i];
    return x;
}

// Squares in fp64: gradients are small enough for their squares to leave the range of fp32.
template <bool BF16, int VEC>
__global__ void __launch_bounds__(256)
square_sum_kernel(const __grid_constant__ PtrTable updates, double* __restrict__ partial, int64_t units)
{
    chain_next();
    chain_wait();
    const void* u = updates.p[blockIdx.y];
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (int64_t)gridDim.x * 256) {
        float v[VEC];
        load_update<BF16, VEC>(u, i, v);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum += (double)v[j] * (double)v[j];
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[(int64_t)blockIdx.y * kNormBlocks + blockIdx.x] = sum;
}

template <bool BF16, int VEC>
__global__ void __launch_bounds__(256)
first_x_kernel(const __grid_constant__ PtrTable updates, const double* __restrict__ partial, int parts, uint16_t* __restrict__ hi,
               uint16_t* __restrict__ lo, int64_t units, uint32_t units_per_row, int64_t ld, int64_t stride, double eps)
{
    chain_next();
    chain_wait();
    const double sum = block_sum((int)threadIdx.x < parts ? partial[(int64_t)blockIdx.y * kNormBlocks + threadIdx.x] : 0.0);
    const double norm = sqrt(sum) + eps;
    const double f = norm > 0.0 ? (double)kX / norm : 0.0;      // not in fp32: 1 / norm of a tiny update leaves its range
    const void* u = updates.p[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (int64_t)gridDim.x * 256) {
        float v[VEC];
        load_update<BF16, VEC>(u, i, v);
        const int64_t row = i / units_per_row;
        const int64_t at = (int64_t)blockIdx.y * stride + row * ld + (i - row * units_per_row) * VEC;
        float x[VEC], rest[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            x[j] = (float)((double)v[j] * f);
            rest[j] = x[j] - __half2float(__float2half_rn(x[j]));
        }
        if constexpr (VEC == 8) {
            *reinterpret_cast<uint4*>(hi + at) = make_uint4(pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7]));
            *reinterpret_cast<uint4*>(lo + at) = make_uint4(pack_f16(rest[0], rest[1]), pack_f16(rest[2], rest[3]), pack_f16(rest[4], rest[5]), pack_f16(rest[6], rest[7]));
        } else {
            hi[at] = (uint16_t)pack_f16(x[0], 0.0f);
            lo[at] = (uint16_t)pack_f16(rest[0], 0.0f);
        }
    }
}

// ------------------------------------------------------------------------------------------------ epilogues

// Symmetric result: scale x acc (+ add x aux), stored at (row, col) and, off the diagonal, at (col, row).
struct SymEpi {
    static constexpr bool kSym = true;
    static constexpr int kStaging = (kRing + 2) * kSlotBytes;      // the ring, and two slots for the mirrored chunks in turn
    using State = AuxRing<1>;
    CUtensorMap map_out;         // boxes of 32 rows x 64 columns, swizzled
    CUtensorMap map_mirror;      // the same array, boxes of 64 rows x 32 columns, not swizzled
    CUtensorMap map_aux;         // fp16, read like map_out
    int has_aux;
    float scale, add;

    __device__ __forceinline__ void prefetch() const
    {
        prefetch_map(&map_out);
        prefetch_map(&map_mirror);
        if (has_aux) prefetch_map(&map_aux);
    }
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape& s, const EpiTile& e, State& ring) const
    {
        ring.start<true>(s, e);
        for (int i = 0; i < kRing - 1; ++i) ring.load<BM, BN, true>(s, e, &map_aux, nullptr, has_aux);
    }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State& ring) const
    {
        const bool mirror = e.col0 + BN <= e.tile.tm * BM;
#pragma unroll 1
        for (int c = 0; c < BN && e.col0 + c < s.n; c += 64) {
            const int n = e.col0 + c;
            const uint32_t slot = ring.slot(e, ring.step, 0);
            if (has_aux && !ring.wait(e)) return false;
            uint32_t packed[32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t* p = packed + 16 * h + 4 * q;
                    if (has_aux) {
                        const uint4 w = slot_read(slot, e.lane, 4 * h + q);
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            p[i] = pack_f16(fmaf(add, f16_lo(u[i]), scale * v[8 * q + 2 * i]), fmaf(add, f16_hi(u[i]), scale * v[8 * q + 2 * i + 1]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] = pack_f16(scale * v[8 * q + 2 * i], scale * v[8 * q + 2 * i + 1]);
                    }
                    slot_write(slot, e.lane, 4 * h + q, p[0], p[1], p[2], p[3]);
                }
            }
            const uint32_t t = e.slots + (uint32_t)((kRing + e.slot) * kSlotBytes);
            if (mirror) {
                // rows of 32 elements (64 bytes): column j of the chunk becomes row j, this lane its element
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const uint32_t at = t + (uint32_t)(2 * j) * 64u + (uint32_t)e.lane * 2u;
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((unsigned short)(packed[j] & 0xFFFFu)) : "memory");
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + 64u), "h"((unsigned short)(packed[j] >> 16)) : "memory");
                }
                e.slot ^= 1;
            }
            fence_async_smem();
            __syncwarp();
            if (e.lane == 0) {
                if (e.row0 < s.m) {
                    tma_store(&map_out, slot, n, e.row0, e.tile.batch);
                    if (mirror) tma_store(&map_mirror, t, e.row0, n, e.tile.batch);
                }
                store_commit();
                store_wait_read<1>();      // the chunk before this one has left: its step and its mirror slot are free
            }
            __syncwarp();
            ring.next();
            ring.load<BM, BN, true>(s, e, &map_aux, nullptr, has_aux);
        }
        return true;
    }
};

// X' = a X + acc: two fp16 words per entry, or after the last step bf16(scale X').
struct StepEpi {
    static constexpr bool kSym = false;
    static constexpr int kStaging = kRing * 2 * kSlotBytes;
    using State = AuxRing<2>;
    CUtensorMap map_hi, map_lo;            // X'
    CUtensorMap map_hi_in, map_lo_in;      // X
    OutTable out;
    float a, scale;
    int last, vec;

    __device__ __forceinline__ void prefetch() const
    {
        prefetch_map(&map_hi_in);
        prefetch_map(&map_lo_in);
        if (!last) {
            prefetch_map(&map_hi);
            prefetch_map(&map_lo);
        }
    }
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape& s, const EpiTile& e, State& ring) const
    {
        ring.start<false>(s, e);
        for (int i = 0; i < kRing - 1; ++i) ring.load<BM, BN, false>(s, e, &map_hi_in, &map_lo_in, 2);
    }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State& ring) const
    {
#pragma unroll 1
        for (int c = 0; c < BN && e.col0 + c < s.n; c += 64) {
            const int n = e.col0 + c;
            const uint32_t hi = ring.slot(e, ring.step, 0), lo = ring.slot(e, ring.step, 1);
            if (!ring.wait(e)) return false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint4 x = slot_read(hi, e.lane, 4 * h + q), y = slot_read(lo, e.lane, 4 * h + q);
                    const uint32_t u[4] = {x.x, x.y, x.z, x.w}, w[4] = {y.x, y.y, y.z, y.w};
                    uint32_t r[4], d[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float g0 = fmaf(a, f16_lo(u[i]) + f16_lo(w[i]), v[8 * q + 2 * i]);
                        const float g1 = fmaf(a, f16_hi(u[i]) + f16_hi(w[i]), v[8 * q + 2 * i + 1]);
                        if (last) {
                            r[i] = pack_b16(scale * g0, scale * g1);
                        } else {
                            r[i] = pack_f16(g0, g1);
                            d[i] = pack_f16(g0 - f16_lo(r[i]), g1 - f16_hi(r[i]));
                        }
                    }
                    slot_write(hi, e.lane, 4 * h + q, r[0], r[1], r[2], r[3]);
                    if (!last) slot_write(lo, e.lane, 4 * h + q, d[0], d[1], d[2], d[3]);
                }
            }
            if (last) {
                // rows of the caller's matrix may have any length: whole rows of the slot by ordinary stores
                __syncwarp();
                uint16_t* o = out.p[e.tile.batch];
#pragma unroll 4
                for (int r0 = 0; r0 < 32; r0 += 4) {
                    const int r = r0 + (e.lane >> 3), q = e.lane & 7;
                    const uint4 w = slot_read(hi, r, q);
                    if (e.row0 + r >= s.m) continue;
                    uint16_t* to = o + (int64_t)(e.row0 + r) * s.n + n + 8 * q;
                    if (vec) {
                        if (n + 8 * q < s.n) *reinterpret_cast<uint4*>(to) = w;
                    } else {
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (n + 8 * q + i < s.n) to[i] = (uint16_t)(i & 1 ? u[i / 2] >> 16 : u[i / 2] & 0xFFFFu);
                    }
                }
                __syncwarp();
            } else {
                fence_async_smem();
                __syncwarp();
                if (e.lane == 0) {
                    if (e.row0 < s.m) {
                        tma_store(&map_hi, hi, n, e.row0, e.tile.batch);
                        tma_store(&map_lo, lo, n, e.row0, e.tile.batch);
                    }
                    store_commit();
                    store_wait_read<1>();      // the chunk before this one has left its step
                }
                __syncwarp();
            }
            ring.next();
            ring.load<BM, BN, false>(s, e, &map_hi_in, &map_lo_in, 2);
        }
        return true;
    }
};

// ------------------------------------------------------------------------------------------------ host

struct Layout {
    int64_t group, ld, sq, sq_ld;
    uint64_t norms, hi[2], lo[2], a, p, total;
};

Layout layout_of(int64_t n, int64_t rows, int64_t cols)
{
    Layout l;
    int64_t fit = kGroupElems / (rows * cols);
    fit = fit < 1 ? 1 : fit > kGroup ? kGroup : fit;
    l.group = n < fit ? n : fit;
    l.ld = (cols + 63) / 64 * 64;
    l.sq = rows < cols ? rows : cols;
    l.sq_ld = (l.sq + 63) / 64 * 64;
    uint64_t at = 0;
    auto take = [&at](uint64_t bytes) { const uint64_t o = at; at += align256(bytes); return o; };
    const uint64_t x = 2ull * (uint64_t)(l.group * rows * l.ld), q = 2ull * (uint64_t)(l.group * l.sq * l.sq_ld);
    l.norms = take(8ull * kNormBlocks * kGroup);
    for (int i = 0; i < 2; ++i) { l.hi[i] = take(x); l.lo[i] = take(x); }
    l.a = take(q);
    l.p = take(q);
    l.total = at;
    return l;
}

// Pairs of CTAs with 256 x 256 tiles, or single CTAs with 128 x 128 ones: rounds over the SMs x cycles per tile.  A 64-deep
// block takes 512 cycles of a pair's tensor cores and about 350 of a single CTA's (256, held up by its shared memory);
// filling and draining a tile's pipeline about 3000.
bool use_pairs(int64_t m, int64_t n, int64_t k, int64_t batch, bool sym, int sms)
{
    const int64_t kb = (k + kBK - 1) / kBK;
    auto tiles = [&](int64_t t) {
        const int64_t a = (m + t - 1) / t, b = (n + t - 1) / t;
        return (sym ? a * (a + 1) / 2 : a * b) * batch;
    };
    const int64_t pairs = sms / 2;
    const int64_t two = (tiles(256) + pairs - 1) / pairs * (kb * 512 + 3000), one = (tiles(128) + sms - 1) / sms * (kb * 350 + 3000);
    return two <= one;
}

template <int CG, int BN, bool MN>
int sym_product(const uint16_t* x, int64_t mn, int64_t k, int64_t batch, int64_t x_ld, int64_t x_stride, uint16_t* out, const Layout& l,
                const uint16_t* aux, float scale, float add, cudaStream_t stream)
{
    CUtensorMap m;
    Shape s;
    SymEpi epi;
    int rc;
    const int64_t stride = l.sq * l.sq_ld;
    if ((rc = make_shape<CG, BN, MN, MN, SymEpi>(&s, false, mn, mn, k, batch, 1, 1)) != CAST_OK) return rc;
    if ((rc = operand_map<MN>(&m, x, mn, k, batch, x_ld, x_stride, 128)) != CAST_OK) return rc;
    CUtensorMap mb = m;
    if (BN / CG != 128 && (rc = operand_map<MN>(&mb, x, mn, k, batch, x_ld, x_stride, BN / CG)) != CAST_OK) return rc;
    if ((rc = make_map(&epi.map_out, out, 2, mn, mn, batch, l.sq_ld, stride, 64, 32, true)) != CAST_OK) return rc;
    if ((rc = make_map(&epi.map_mirror, out, 2, mn, mn, batch, l.sq_ld, stride, 32, 64, false)) != CAST_OK) return rc;
    epi.has_aux = aux != nullptr;
    epi.map_aux = epi.map_out;
    if (aux && (rc = make_map(&epi.map_aux, aux, 2, mn, mn, batch, l.sq_ld, stride, 64, 32, true)) != CAST_OK) return rc;
    epi.scale = scale;
    epi.add = add;
    return launch<CG, BN, MN, MN>(m, mb, s, epi, stream);
}

// X' = a X + P X (wide) or a X + X P (tall)
template <int CG, int BN, bool WIDE>
int step_product(const uint16_t* p, const uint16_t* hi, const uint16_t* lo, int64_t rows, int64_t cols, int64_t batch, const Layout& l, uint16_t* hi_out,
                 uint16_t* lo_out, StepEpi& epi, cudaStream_t stream)
{
    CUtensorMap ma, mb;
    Shape s;
    int rc;
    const int64_t xs = rows * l.ld, ps = l.sq * l.sq_ld;
    if ((rc = make_shape<CG, BN, false, WIDE, StepEpi>(&s, false, rows, cols, l.sq, batch, 1, 16 / CG)) != CAST_OK) return rc;
    if (WIDE) {
        if ((rc = operand_map<false>(&ma, p, rows, rows, batch, l.sq_ld, ps, 128)) != CAST_OK) return rc;
        if ((rc = operand_map<true>(&mb, hi, cols, rows, batch, l.ld, xs, BN / CG)) != CAST_OK) return rc;
    } else {
        if ((rc = operand_map<false>(&ma, hi, rows, cols, batch, l.ld, xs, 128)) != CAST_OK) return rc;
        if ((rc = operand_map<false>(&mb, p, cols, cols, batch, l.sq_ld, ps, BN / CG)) != CAST_OK) return rc;
    }
    if ((rc = make_map(&epi.map_hi, hi_out, 2, cols, rows, batch, l.ld, xs, 64, 32, true)) != CAST_OK) return rc;
    if ((rc = make_map(&epi.map_lo, lo_out, 2, cols, rows, batch, l.ld, xs, 64, 32, true)) != CAST_OK) return rc;
    if ((rc = make_map(&epi.map_hi_in, hi, 2, cols, rows, batch, l.ld, xs, 64, 32, true)) != CAST_OK) return rc;
    if ((rc = make_map(&epi.map_lo_in, lo, 2, cols, rows, batch, l.ld, xs, 64, 32, true)) != CAST_OK) return rc;
    return launch<CG, BN, false, WIDE>(ma, mb, s, epi, stream);
}

template <bool BF16, int VEC>
int launch_first(bool first, const PtrTable& t, int64_t batch, int64_t rows, int64_t cols, uint8_t* ws, const Layout& l, float eps, cudaStream_t stream)
{
    const int64_t units = rows * cols / VEC;
    int64_t parts = (units + 256 * 8 - 1) / (256 * 8);
    if (parts > kNormBlocks) parts = kNormBlocks;
    double* norms = reinterpret_cast<double*>(ws + l.norms);
    int rc = launch_chained(first, square_sum_kernel<BF16, VEC>, dim3((unsigned)parts, (unsigned)batch), 256, 0, stream, 1, t, norms, units);
    if (rc != CAST_OK) return rc;
    int64_t blocks = (units + 256 * 4 - 1) / (256 * 4);
    if (blocks > 2048) blocks = 2048;
    return launch_chained(false, first_x_kernel<BF16, VEC>, dim3((unsigned)blocks, (unsigned)batch), 256, 0, stream, 1, t, norms, (int)parts,
                          reinterpret_cast<uint16_t*>(ws + l.hi[0]), reinterpret_cast<uint16_t*>(ws + l.lo[0]), units, (uint32_t)(cols / VEC), l.ld,
                          rows * l.ld, (double)eps);
}

int check_ortho_shape(int64_t n, int64_t rows, int64_t cols)
{
    if (n < 1 || rows < 1 || cols < 1 || n > 0x7FFFFFFF) return CAST_ERR_SHAPE;
    if (rows > 0x7FFFFFFF / cols) return CAST_ERR_SHAPE;      // rows*cols < 2^31, as for every matrix of the library
    return CAST_OK;
}

// No result shares memory with an update or another result: the ranges in address order, against the furthest end so far.
int check_apart(const void* const* updates, uint64_t in_bytes, cast_bf16* const* out, uint64_t out_bytes, int n)
{
    struct Range { uintptr_t lo, hi; bool result; };
    Range few[64];
    Range* r = 2 * (int64_t)n <= 64 ? few : new (std::nothrow) Range[2 * (size_t)n];
    if (!r) return CAST_ERR_MEMORY;
    for (int i = 0; i < n; ++i) {
        const uintptr_t u = (uintptr_t)updates[i], o = (uintptr_t)out[i];
        r[2 * i] = {u, u + in_bytes, false};
        r[2 * i + 1] = {o, o + out_bytes, true};
    }
    std::sort(r, r + 2 * (size_t)n, [](const Range& a, const Range& b) { return a.lo < b.lo; });
    uintptr_t any = 0, result = 0;
    int rc = CAST_OK;
    for (size_t i = 0; i < 2 * (size_t)n; ++i) {
        if (r[i].lo < (r[i].result ? any : result)) rc = CAST_ERR_ALIAS;
        any = std::max(any, r[i].hi);
        if (r[i].result) result = std::max(result, r[i].hi);
    }
    if (r != few) delete[] r;
    return rc;
}

}  // namespace
}  // namespace cast

using namespace cast;

extern "C" int cast_orthogonalize_workspace(int n, int64_t rows, int64_t cols, uint64_t* bytes)
{
    if (!bytes) return CAST_ERR_NULL;
    int rc;
    if ((rc = check_ortho_shape(n, rows, cols)) != CAST_OK) return rc;
    *bytes = layout_of(n, rows, cols).total;
    return CAST_OK;
}

extern "C" int cast_orthogonalize(const void* const* updates, int updates_bf16, cast_bf16* const* out, int n, int64_t rows, int64_t cols,
                                  const float* coeffs, int steps, float eps, float scale, void* workspace, uint64_t workspace_bytes,
                                  cast_stream_t stream)
{
    static const float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
    if (!updates || !out || !workspace) return CAST_ERR_NULL;
    int rc, sms;
    if ((rc = check_ortho_shape(n, rows, cols)) != CAST_OK) return rc;
    if (steps < 1 || steps > 100 || !(eps >= 0.0f) || !std::isfinite(eps) || !std::isfinite(scale)) return CAST_ERR_HYPER;
    for (int i = 0; coeffs && i < 3 * steps; ++i)
        if (!std::isfinite(coeffs[i])) return CAST_ERR_HYPER;
    if ((uintptr_t)workspace & 15u) return CAST_ERR_ALIGN;
    const Layout l = layout_of(n, rows, cols);
    if (workspace_bytes < l.total) return CAST_ERR_PLAN;
    const uintptr_t mask = updates_bf16 ? 1u : 3u;
    const uint64_t in_bytes = (updates_bf16 ? 2ull : 4ull) * (uint64_t)(rows * cols), out_bytes = 2ull * (uint64_t)(rows * cols);
    for (int i = 0; i < n; ++i) {
        if (!updates[i] || !out[i]) return CAST_ERR_NULL;
        if (((uintptr_t)updates[i] & mask) || ((uintptr_t)out[i] & 1u)) return CAST_ERR_ALIGN;
        if (ranges_overlap(workspace, l.total, updates[i], in_bytes) || ranges_overlap(workspace, l.total, out[i], out_bytes)) return CAST_ERR_ALIAS;
    }
    if ((rc = check_apart(updates, in_bytes, out, out_bytes, n)) != CAST_OK) return rc;
    if ((rc = check_device_memory(updates, n)) != CAST_OK) return rc;
    if ((rc = check_device_memory(reinterpret_cast<const void* const*>(out), n)) != CAST_OK) return rc;
    if ((rc = check_device_memory(&workspace, 1)) != CAST_OK) return rc;
    if ((rc = product::sm_count(&sms)) != CAST_OK) return rc;

    uint8_t* ws = static_cast<uint8_t*>(workspace);
    cudaStream_t st = (cudaStream_t)stream;
    const bool wide = rows <= cols;
    const int64_t big = wide ? cols : rows;
    uint16_t* hi[2] = {reinterpret_cast<uint16_t*>(ws + l.hi[0]), reinterpret_cast<uint16_t*>(ws + l.hi[1])};
    uint16_t* lo[2] = {reinterpret_cast<uint16_t*>(ws + l.lo[0]), reinterpret_cast<uint16_t*>(ws + l.lo[1])};
    uint16_t* a = reinterpret_cast<uint16_t*>(ws + l.a);
    uint16_t* p = reinterpret_cast<uint16_t*>(ws + l.p);
    for (int first = 0; first < n; first += (int)l.group) {
        const int64_t batch = n - first < l.group ? n - first : l.group;
        PtrTable in;
        StepEpi epi;
        bool in_vec = cols % 8 == 0, out_vec = cols % 8 == 0;
        for (int64_t i = 0; i < batch; ++i) {
            in.p[i] = updates[first + i];
            epi.out.p[i] = out[first + i];
            in_vec = in_vec && !((uintptr_t)in.p[i] & 15u);
            out_vec = out_vec && !((uintptr_t)epi.out.p[i] & 15u);
        }
        for (int64_t i = batch; i < kGroup; ++i) { in.p[i] = nullptr; epi.out.p[i] = nullptr; }
        if (updates_bf16) rc = in_vec ? launch_first<true, 8>(first == 0, in, batch, rows, cols, ws, l, eps, st) : launch_first<true, 1>(first == 0, in, batch, rows, cols, ws, l, eps, st);
        else rc = in_vec ? launch_first<false, 8>(first == 0, in, batch, rows, cols, ws, l, eps, st) : launch_first<false, 1>(first == 0, in, batch, rows, cols, ws, l, eps, st);
        if (rc != CAST_OK) return rc;
        const bool gram2 = use_pairs(l.sq, l.sq, big, batch, true, sms), sq2 = use_pairs(l.sq, l.sq, l.sq, batch, true, sms);
        const bool step2 = use_pairs(rows, cols, l.sq, batch, false, sms);
        const float down = 1.0f / (kX * kX);
        for (int k = 0; k < steps; ++k) {
            const float* q = coeffs ? coeffs + 3 * k : kQuintic;
            const int cur = k & 1;
            const int64_t xs = rows * l.ld, ps = l.sq * l.sq_ld;
            if (wide) rc = gram2 ? sym_product<2, 256, false>(hi[cur], rows, cols, batch, l.ld, xs, a, l, nullptr, down, 0.0f, st)
                                 : sym_product<1, 128, false>(hi[cur], rows, cols, batch, l.ld, xs, a, l, nullptr, down, 0.0f, st);
            else rc = gram2 ? sym_product<2, 256, true>(hi[cur], cols, rows, batch, l.ld, xs, a, l, nullptr, down, 0.0f, st)
                            : sym_product<1, 128, true>(hi[cur], cols, rows, batch, l.ld, xs, a, l, nullptr, down, 0.0f, st);
            if (rc != CAST_OK) return rc;
            rc = sq2 ? sym_product<2, 256, false>(a, l.sq, l.sq, batch, l.sq_ld, ps, p, l, a, q[2], q[1], st)
                     : sym_product<1, 128, false>(a, l.sq, l.sq, batch, l.sq_ld, ps, p, l, a, q[2], q[1], st);
            if (rc != CAST_OK) return rc;
            epi.a = q[0];
            epi.scale = scale / kX;
            epi.last = k + 1 == steps;
            epi.vec = out_vec;
            if (wide) rc = step2 ? step_product<2, 256, true>(p, hi[cur], lo[cur], rows, cols, batch, l, hi[cur ^ 1], lo[cur ^ 1], epi, st)
                                 : step_product<1, 128, true>(p, hi[cur], lo[cur], rows, cols, batch, l, hi[cur ^ 1], lo[cur ^ 1], epi, st);
            else rc = step2 ? step_product<2, 256, false>(p, hi[cur], lo[cur], rows, cols, batch, l, hi[cur ^ 1], lo[cur ^ 1], epi, st)
                            : step_product<1, 128, false>(p, hi[cur], lo[cur], rows, cols, batch, l, hi[cur ^ 1], lo[cur ^ 1], epi, st);
            if (rc != CAST_OK) return rc;
        }
    }
    return CAST_OK;
}
