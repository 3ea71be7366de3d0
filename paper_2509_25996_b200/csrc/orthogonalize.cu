// Newton-Schulz orthogonalisation of updates (as the Muon optimiser applies it to hidden matrices):
//     X = U / (|U|_F + eps),   steps times  X <- a X + (b A + c A A) X,  A = X X^T,   out = scale X
// and X <- a X + X (b A + c A A) with A = X^T X where there are more rows than columns, so that A is the smaller square.
//
// Each step is three products on the tensor cores over all matrices of the call at once:
//     A = X X^T               symmetric: only tiles on and below the diagonal, each stored twice (once transposed)
//     P = a I + b A + c A A   symmetric likewise; a I + b A is added by the epilogue
//     X' = P X
// A long and narrow X gives A few tiles with a long sum each: its k is then cut into splits whose fp32 sums a small kernel adds.
// Operands are never transposed in memory: X is read K-major in one product and MN-major in the other.
//
// Numbers: the operands are fp16, not bf16.  Every value is bounded (|X| singular values stay near 1), so the range is
// enough and the 3 more bits of significand are worth 8 times less rounding noise.  Noise of A and P enters through directions
// that are large already; what remains of it is P's diagonal, rounded alike in every step (~1e-3 of the result).  Rounding X itself
// is worse: that noise lies in all directions, and a step multiplies small ones by a = 3.4, five steps by 500, which swamps an
// update of low rank (measured on 768 x 768 of rank 8 over 2 % noise: 2.8e-2 from the exact result, where rounding the result to
// bf16 is 1.7e-3).  So while the steps still to come amplify by more than kAmplify, X is held as hi + lo, two fp16 words scaled by
// 2^12 (22 bits); with five steps X_0 (of an fp32 update; a bf16 one is exact in hi) to X_3 have a lo.  The products read hi;
// P lo is replaced by kappa lo, kappa the mean of P's diagonal: rounding noise has no direction, so that is the nearest multiple
// of lo to P lo.  It is a for an update of low rank, and near 1 where most directions have grown: there a lo would be further
// from P lo than nothing is.  |out - exact| / |exact| for 768 x 768 without structure / of low rank, kAmplify 12 with a lo:
// 2.00e-3 / 2.55e-3; 4 with a lo: 2.08e-3 / 1.92e-3; 4 with kappa lo: 1.98e-3 / 1.92e-3.
//
// What bounds it: for large matrices the tensor cores at the clock that the power limit leaves them (4096 x 11008: 2.77 ms, 1.13
// PFLOP/s counting symmetric products by half); for twelve 3072 x 768 matrices (522 us) the path from L2 to the SMs, which
// feeds a pair's tile 64 bytes per cycle and SM, just as much as it consumes, and X and its two words, which exceed L2; for one
// 768 x 768 (93 us) the chain of 17 kernels, of ~5.4 us each: 1 us until the first operands are there, 1.8 us of products, 1 us
// of epilogue, 1.5 us until its successor sees the results.
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
constexpr int64_t kGroupElems = 64 << 20;   // ... and elements of padded rows, which bounds the workspace
constexpr int kNormBlocks = 1024;           // per matrix at most
// X keeps its lo while later steps multiply small directions by more.  One word of X_4 amplified by 3.4 is 7e-4 of the result
// at most, of X_3 2.5e-3, more than the result's own rounding.  Keeping X_3's and kappa take twelve
// 3072 x 768 from 501 to 520 us, one 768 x 768 from 91.2 to 93.3.
constexpr float kAmplify = 4.0f;

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

// Sum of squares of a matrix from its CTAs' parts, by every CTA that needs it, in the same order.
__device__ __forceinline__ double total_of(const double* part, int parts)
{
    double sum = 0.0;
    for (int i = (int)threadIdx.x; i < parts; i += 256) sum += part[i];
    return block_sum(sum);
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

// X_0, stored times kX.  A bf16 update keeps its significands: it is scaled by a power of two, hi is exact, there is no lo, and
// the rest of the scale, gain[matrix] in [1, 2), is applied by the first step's epilogues.
template <bool BF16, int VEC>
__global__ void __launch_bounds__(256)
first_x_kernel(const __grid_constant__ PtrTable updates, const double* __restrict__ partial, int parts, uint16_t* __restrict__ hi,
               uint16_t* __restrict__ lo, float* __restrict__ gain, int64_t units, uint32_t units_per_row, int64_t ld, int64_t stride, double eps)
{
    chain_next();
    chain_wait();
    const double norm = sqrt(total_of(partial + (int64_t)blockIdx.y * kNormBlocks, parts)) + eps;
    double f = norm > 0.0 ? (double)kX / norm : 0.0;      // not in fp32: 1 / norm of a tiny update leaves its range
    if constexpr (BF16) {
        int e = 0;
        const double g = f > 0.0 ? 2.0 * frexp(f, &e) : 1.0;
        f = f > 0.0 ? ldexp(1.0, e - 1) : 0.0;
        if (blockIdx.x == 0 && threadIdx.x == 0) gain[blockIdx.y] = (float)g;
    }
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
            if constexpr (!BF16)
                *reinterpret_cast<uint4*>(lo + at) = make_uint4(pack_f16(rest[0], rest[1]), pack_f16(rest[2], rest[3]), pack_f16(rest[4], rest[5]), pack_f16(rest[6], rest[7]));
        } else {
            hi[at] = (uint16_t)pack_f16(x[0], 0.0f);
            if constexpr (!BF16) lo[at] = (uint16_t)pack_f16(rest[0], 0.0f);
        }
    }
}

// ------------------------------------------------------------------------------------------------ epilogues

// Mean of the diagonal of a matrix's P, by a converged warp, in the same order everywhere.
__device__ __forceinline__ float mean_diagonal(const float* traces, int batch, int n)
{
    const int blocks = (n + 31) / 32;
    float sum = 0.0f;
    for (int i = (int)threadIdx.x & 31; i < blocks; i += 32) sum += __ldg(traces + (int64_t)batch * blocks + i);
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k);
    return sum / (float)n;
}

// The ring of lo, and kappa of the matrix at hand.
struct LoState {
    AuxRing ring;
    int batch;
    float kappa;
    __device__ __forceinline__ void find_kappa(const float* traces, int of, int n)
    {
        if (of == batch) return;
        batch = of;
        kappa = mean_diagonal(traces, of, n);
    }
};

// A symmetric result, stored at (row, col) and, off the diagonal, at (col, row): scale acc, or with POLY
// scale acc + add aux + diag I.
template <bool POLY>
struct SymEpi {
    static constexpr bool kSym = true;
    static constexpr bool kInputsOnly = false;
    static constexpr int kRunStages = 0;
    // eight with a ring would leave the products four stages instead of five: twelve 3072 x 768 500 -> 495 us, but 4096 x 11008
    // 2700 -> 2720 and 768 x 768 92.6 -> 93.2; with StepEpi's likewise 2750
    static constexpr int kWarps = POLY ? 4 : 8;
    // POLY: the ring of aux, replaced in place, and a slot for the mirrored chunk; otherwise a slot for each
    static constexpr int kStaging = (POLY ? kRing + 1 : 2) * kSlotBytes;
    using State = AuxRing;
    CUtensorMap map_out;         // boxes of 32 rows x 64 columns, swizzled
    CUtensorMap map_mirror;      // the same array, boxes of 64 rows x 32 columns, not swizzled
    CUtensorMap map_aux;         // fp16, read like map_out
    const float* gain;           // per matrix, its square multiplies the result; nullptr: 1
    float* traces;               // POLY: [batch][blocks], sums of the diagonal over blocks of 32
    float scale, add, diag;

    __device__ __forceinline__ void prefetch() const
    {
        prefetch_map(&map_out);
        prefetch_map(&map_mirror);
        if constexpr (POLY) prefetch_map(&map_aux);
    }
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape& s, const EpiTile& e, State& ring) const
    {
        if constexpr (POLY) {
            ring.start<BN, true>(s, e);
            for (int i = 0; i < kRing - 1; ++i) ring.load<BM, BN, true>(s, e, &map_aux);
        }
    }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State& ring) const
    {
        const bool mirror = e.col0 + BN <= e.tile.tm * BM;
        const float g = gain ? __ldg(gain + e.tile.batch) : 1.0f, scale_all = scale * g * g;
        [[maybe_unused]] float on_diagonal = 0.0f;
#pragma unroll 1
        for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 64) {
            const int n = e.col0 + c;
            slots_free(e);
            uint32_t slot = e.slots;
            if constexpr (POLY) {
                ring.load<BM, BN, true>(s, e, &map_aux);
                slot = ring.slot(e);
                if (!ring.wait(e)) return false;
            }
            const uint32_t t = e.slots + (uint32_t)((POLY ? kRing : 1) * kSlotBytes);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {      // a loop: half the code to fetch in a kernel that runs a few microseconds
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= scale_all;
                if constexpr (POLY) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint4 w = slot_read(slot, e.lane, 4 * h + q);
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            v[8 * q + 2 * i] = fmaf(add, f16_lo(u[i]), v[8 * q + 2 * i]);
                            v[8 * q + 2 * i + 1] = fmaf(add, f16_hi(u[i]), v[8 * q + 2 * i + 1]);
                        }
                    }
                    // (no branch around this: the few warps that meet the diagonal would fetch its code for ~1500 cycles)
                    const int d = e.row0 + e.lane - (n + 32 * h);      // where this row's diagonal entry lies in these columns
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] += i == d ? diag : 0.0f;
                }
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i] = pack_f16(v[2 * i], v[2 * i + 1]);
#pragma unroll
                for (int q = 0; q < 4; ++q) slot_write(slot, e.lane, 4 * h + q, p[4 * q], p[4 * q + 1], p[4 * q + 2], p[4 * q + 3]);
                if constexpr (POLY) {
                    // a lane's own entry of the diagonal, where these 32 rows and columns are the same ones (no branch, as above)
                    const float own = f16_lo(slot_read_16(slot, e.lane, 32 * h + e.lane));
                    on_diagonal = e.row0 == n + 32 * h && e.row0 + e.lane < s.m ? own : on_diagonal;
                }
                if (mirror) {
                    // rows of 32 elements (64 bytes): column j of the chunk becomes row j, this lane its element
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t at = t + (uint32_t)(32 * h + 2 * j) * 64u + (uint32_t)e.lane * 2u;
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((unsigned short)(p[j] & 0xFFFFu)) : "memory");
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + 64u), "h"((unsigned short)(p[j] >> 16)) : "memory");
                    }
                }
            }
            fence_async_smem();
            __syncwarp();
            if (e.lane == 0) {
                if (e.row0 < s.m) {
                    tma_store(&map_out, slot, n, e.row0, e.tile.batch);
                    if (mirror) tma_store(&map_mirror, t, e.row0, n, e.tile.batch);
                }
                store_commit();
            }
            if constexpr (POLY) ring.next();
        }
        if constexpr (POLY) {
#pragma unroll
            for (int k = 16; k > 0; k >>= 1) on_diagonal += __shfl_xor_sync(0xFFFFFFFFu, on_diagonal, k);
            const int first = e.col0 + e.c0;
            if (e.lane == 0 && e.row0 >= first && e.row0 < min(s.m, first + e.c1 - e.c0))
                traces[(int64_t)e.tile.batch * ((s.m + 31) / 32) + e.row0 / 32] = on_diagonal;
        }
        return true;
    }
};

// One split's sums of A as they are, fp32 [matrix][split][row][column]; blocks above the diagonal are left out.
struct PartEpi {
    static constexpr bool kSym = true;
    static constexpr bool kInputsOnly = false;
    static constexpr int kRunStages = 0;
    static constexpr int kWarps = 8;
    static constexpr int kStaging = kSlotBytes;
    struct State {};
    CUtensorMap map_out;

    __device__ __forceinline__ void prefetch() const { prefetch_map(&map_out); }
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape&, const EpiTile&, State&) const {}

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State&) const
    {
#pragma unroll 1
        for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 32) {
            float v[32];
            const uint32_t slot = slot_acquire(e);
            tmem_load32(e.acc + (uint32_t)c, v);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                slot_write(slot, e.lane, q, __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
            slot_store(e, slot, &map_out, e.col0 + c, e.row0, e.tile.batch * s.splits + e.tile.split, e.row0 < s.m);
        }
        return true;
    }
};

// A = scale gain^2 (sum of the splits, in order): a CTA takes one 32 x 32 block on or below the diagonal and stores it twice.
__global__ void __launch_bounds__(256)
add_parts_kernel(const float* __restrict__ parts, uint16_t* __restrict__ out, const float* __restrict__ gain, int splits, int n, int64_t part_ld, int64_t ld,
                 float scale)
{
    __shared__ uint16_t block[32][33];
    chain_next();
    chain_wait();
    int row = (int)((sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
    while (row * (row + 1) / 2 > (int)blockIdx.x) --row;
    while ((row + 1) * (row + 2) / 2 <= (int)blockIdx.x) ++row;
    const int r0 = 32 * row, c0 = 32 * ((int)blockIdx.x - row * (row + 1) / 2);
    const int r = (int)threadIdx.x >> 3, c = ((int)threadIdx.x & 7) * 4;        // four columns of a row
    const float g = gain ? __ldg(gain + blockIdx.y) : 1.0f, by = scale * g * g;
    const int64_t size = (int64_t)n * part_ld;
    if (r0 + r < n) {
        // rows are padded to whole vectors; what lies past the last column is not stored
        const float* p = parts + (int64_t)blockIdx.y * splits * size + (int64_t)(r0 + r) * part_ld + c0 + c;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int s0 = 0; s0 < splits; s0 += 8) {
            float4 x[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = s0 + s < splits ? __ldg(reinterpret_cast<const float4*>(p + (s0 + s) * size)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int s = 0; s < 8; ++s) { sum.x += x[s].x; sum.y += x[s].y; sum.z += x[s].z; sum.w += x[s].w; }
        }
        const uint32_t lo = pack_f16(by * sum.x, by * sum.y), hi = pack_f16(by * sum.z, by * sum.w);
        block[r][c] = (uint16_t)(lo & 0xFFFFu);
        block[r][c + 1] = (uint16_t)(lo >> 16);
        block[r][c + 2] = (uint16_t)(hi & 0xFFFFu);
        block[r][c + 3] = (uint16_t)(hi >> 16);
    }
    __syncthreads();
    uint16_t* o = out + (int64_t)blockIdx.y * n * ld;
    for (int i = threadIdx.x; i < 1024; i += 256) {
        const int y = i >> 5, x = i & 31;
        if (r0 + y < n && c0 + x < n) o[(int64_t)(r0 + y) * ld + c0 + x] = block[y][x];
        if (r0 != c0 && r0 + x < n && c0 + y < n) o[(int64_t)(c0 + y) * ld + r0 + x] = block[x][y];
    }
}

// X' = gain acc (+ kappa lo): as hi + lo, or hi alone.
template <bool LO_IN, bool LO_OUT>
struct StepEpi {
    static constexpr bool kSym = false;
    static constexpr bool kInputsOnly = false;
    static constexpr int kRunStages = 0;
    static constexpr int kWarps = LO_IN ? 4 : 8;
    // LO_IN: the ring of lo, replaced in place by the new one, and a slot for hi; otherwise a slot for each
    static constexpr int kStaging = (LO_IN ? kRing + 1 : LO_OUT ? 2 : 1) * kSlotBytes;
    using State = LoState;
    CUtensorMap map_hi, map_lo;      // X'
    CUtensorMap map_lo_in;           // X
    const float* gain;               // per matrix; nullptr: 1 (only without LO_IN)
    const float* traces;             // of P (LO_IN)
    int sq;

    __device__ __forceinline__ void prefetch() const
    {
        prefetch_map(&map_hi);
        if constexpr (LO_IN) prefetch_map(&map_lo_in);
        if constexpr (LO_OUT) prefetch_map(&map_lo);
    }
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape& s, const EpiTile& e, State& state) const
    {
        if constexpr (LO_IN) {
            state.ring.start<BN, false>(s, e);
            for (int i = 0; i < kRing - 1; ++i) state.ring.load<BM, BN, false>(s, e, &map_lo_in);
            state.batch = -1;
            state.find_kappa(traces, tile_of<false>(s, e.index).batch, sq);
        }
    }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State& state) const
    {
        AuxRing& ring = state.ring;
        if constexpr (LO_IN) state.find_kappa(traces, e.tile.batch, sq);
        float g = 1.0f;
        if constexpr (!LO_IN) g = gain ? __ldg(gain + e.tile.batch) : 1.0f;
#pragma unroll 1
        for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 64) {
            const int n = e.col0 + c;
            uint32_t hi, lo = 0;
            if constexpr (LO_IN) {
                slots_free(e);
                ring.load<BM, BN, false>(s, e, &map_lo_in);
                hi = e.slots + kRing * kSlotBytes;
                lo = ring.slot(e);
                if (!ring.wait(e)) return false;
            } else if constexpr (LO_OUT) {
                slots_free(e);
                hi = e.slots;
                lo = e.slots + kSlotBytes;
            } else {
                hi = slot_acquire(e);
            }
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {      // a loop: half the code to fetch in a kernel that runs a few microseconds
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t w[4] = {0u, 0u, 0u, 0u}, r[4], d[4];
                    if constexpr (LO_IN) {
                        const uint4 y = slot_read(lo, e.lane, 4 * h + q);
                        w[0] = y.x; w[1] = y.y; w[2] = y.z; w[3] = y.w;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float g0 = v[8 * q + 2 * i], g1 = v[8 * q + 2 * i + 1];
                        if constexpr (LO_IN) {
                            g0 = fmaf(state.kappa, f16_lo(w[i]), g0);
                            g1 = fmaf(state.kappa, f16_hi(w[i]), g1);
                        } else {
                            g0 *= g;
                            g1 *= g;
                        }
                        r[i] = pack_f16(g0, g1);
                        if constexpr (LO_OUT) d[i] = pack_f16(g0 - f16_lo(r[i]), g1 - f16_hi(r[i]));
                    }
                    slot_write(hi, e.lane, 4 * h + q, r[0], r[1], r[2], r[3]);
                    if constexpr (LO_OUT) slot_write(lo, e.lane, 4 * h + q, d[0], d[1], d[2], d[3]);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (e.lane == 0) {
                if (e.row0 < s.m) {
                    tma_store(&map_hi, hi, n, e.row0, e.tile.batch);
                    if constexpr (LO_OUT) tma_store(&map_lo, lo, n, e.row0, e.tile.batch);
                }
                store_commit();
            }
            if constexpr (LO_IN) ring.next();
        }
        return true;
    }
};

// The result: bf16(scale (acc + kappa lo)) into the caller's matrices, whose rows may have any length and alignment: through a slot,
// then whole rows of it by ordinary stores.
template <bool LO_IN>
struct ResultEpi {
    static constexpr bool kSym = false;
    static constexpr bool kInputsOnly = false;
    static constexpr int kRunStages = 0;
    static constexpr int kWarps = LO_IN ? 4 : 8;
    static constexpr int kStaging = (LO_IN ? kRing : 1) * kSlotBytes;
    using State = LoState;
    CUtensorMap map_lo_in;
    OutTable out;
    const float* gain;               // as in StepEpi
    const float* traces;
    float scale;
    int sq, vec;

    __device__ __forceinline__ void prefetch() const { if constexpr (LO_IN) prefetch_map(&map_lo_in); }
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape& s, const EpiTile& e, State& state) const
    {
        if constexpr (LO_IN) {
            state.ring.start<BN, false>(s, e);
            for (int i = 0; i < kRing - 1; ++i) state.ring.load<BM, BN, false>(s, e, &map_lo_in);
            state.batch = -1;
            state.find_kappa(traces, tile_of<false>(s, e.index).batch, sq);
        }
    }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State& state) const
    {
        AuxRing& ring = state.ring;
        if constexpr (LO_IN) state.find_kappa(traces, e.tile.batch, sq);
        uint16_t* o = out.p[e.tile.batch];
        float by = scale;
        if constexpr (!LO_IN) by *= gain ? __ldg(gain + e.tile.batch) : 1.0f;
#pragma unroll 1
        for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 64) {
            const int n = e.col0 + c;
            // the chunk before this one has been read; its slot, which ordinary stores have written, is the one that is loaded next
            if constexpr (LO_IN) fence_async_smem();
            __syncwarp();
            uint32_t slot = e.slots;
            if constexpr (LO_IN) {
                ring.load<BM, BN, false>(s, e, &map_lo_in);
                slot = ring.slot(e);
                if (!ring.wait(e)) return false;
            }
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {      // a loop: half the code to fetch in a kernel that runs a few microseconds
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (LO_IN) {
                        const uint4 y = slot_read(slot, e.lane, 4 * h + q);
                        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            v[8 * q + 2 * i] = fmaf(state.kappa, f16_lo(w[i]), v[8 * q + 2 * i]);
                            v[8 * q + 2 * i + 1] = fmaf(state.kappa, f16_hi(w[i]), v[8 * q + 2 * i + 1]);
                        }
                    }
                    slot_write(slot, e.lane, 4 * h + q, pack_b16(by * v[8 * q], by * v[8 * q + 1]),
                               pack_b16(by * v[8 * q + 2], by * v[8 * q + 3]), pack_b16(by * v[8 * q + 4], by * v[8 * q + 5]),
                               pack_b16(by * v[8 * q + 6], by * v[8 * q + 7]));
                }
            }
            __syncwarp();
#pragma unroll 4
            for (int r0 = 0; r0 < 32; r0 += 4) {
                const int r = r0 + (e.lane >> 3), q = e.lane & 7;
                const uint4 w = slot_read(slot, r, q);
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
            if constexpr (LO_IN) ring.next();
        }
        return true;
    }
};

// ------------------------------------------------------------------------------------------------ host

enum TileForm { kPair256, kSingle128, kSingle64 };      // 256 x 256 on two CTAs, 128 x 128 or 128 x 64 on one

constexpr int kSms = 148;                                // the choice goes by a B200's, so that the workspace's size does not depend on the device
constexpr int kMostSplits = 16;
constexpr int64_t kPartBytes = 64 << 20;                 // of fp32 sums at most

struct Form { TileForm tile; int splits; };

// The form that takes least: rounds over the SMs x cycles per tile.  A 64-deep block of a pair's 256 x 256 takes 512 cycles of its
// tensor cores; a single CTA is bound by its L2 port, 64 bytes per cycle: 512 cycles for 32 KB (128 x 128), 384 for 24 KB
// (128 x 64).  Filling and draining a tile's pipeline: about 3000 cycles and 16 per column of its epilogue.  Splits of k (symmetric
// products only) cost another kernel, about 8000 cycles, and their sums written and read at ~2.5 KB per cycle.  (Measured from
// 256 x 256 to 4096 x 4096, alone and in batches: no other tile is more than 3 % faster than the one chosen.  The cycles are those
// of operands in L2, the same for all forms where they are not: the choice goes by their order, not by their sum.)
Form choose_form(int64_t m, int64_t n, int64_t k, int64_t batch, bool sym, int most_splits = kMostSplits)
{
    const int64_t kb = (k + kBK - 1) / kBK;
    Form best = {kPair256, 1};
    int64_t least = INT64_MAX;
    for (int s = 1; s <= most_splits && s <= kb; ++s) {
        if (s > 1 && 4 * s * batch * m * ((n + 63) / 64 * 64) > kPartBytes) break;
        auto consider = [&](TileForm f, int64_t bm, int64_t bn, int64_t units, int64_t block) {
            const int64_t a = (m + bm - 1) / bm, b = (n + bn - 1) / bn;
            const int64_t tiles = (sym ? a * (a + 1) / 2 * (bm / bn) : a * b) * batch * s;
            int64_t cost = (tiles + units - 1) / units * ((kb + s - 1) / s * block) + 3000 + 16 * bn;
            if (s > 1) cost += 8000 + 8 * s * batch * m * n / 2500;
            if (cost < least) { least = cost; best = {f, s}; }
        };
        consider(kPair256, 256, 256, kSms / 2, 512);
        consider(kSingle128, 128, 128, kSms, 512);
        consider(kSingle64, 128, 64, kSms, 384);
    }
    return best;
}

struct Layout {
    int64_t group, ld, sq, sq_ld;
    uint64_t norms, gains, traces, hi[2], lo[2], a, p, parts, total;
};

Layout layout_of(int64_t n, int64_t rows, int64_t cols)
{
    Layout l;
    // whole 128-byte lines per row, or where a row is shorter than one the 16 bytes that a copy needs
    l.ld = cols < 64 ? (cols + 7) / 8 * 8 : (cols + 63) / 64 * 64;
    int64_t fit = kGroupElems / (rows * l.ld);
    fit = fit < 1 ? 1 : fit > kGroup ? kGroup : fit;
    l.group = n < fit ? n : fit;
    l.sq = rows < cols ? rows : cols;
    l.sq_ld = (l.sq + 63) / 64 * 64;
    uint64_t at = 0;
    auto take = [&at](uint64_t bytes) { const uint64_t o = at; at += align256(bytes); return o; };
    const uint64_t x = 2ull * (uint64_t)(l.group * rows * l.ld), q = 2ull * (uint64_t)(l.group * l.sq * l.sq_ld);
    l.norms = take(8ull * kNormBlocks * (uint64_t)l.group);
    l.gains = take(4ull * (uint64_t)l.group);
    l.traces = take(4ull * (uint64_t)(l.group * ((l.sq + 31) / 32)));
    for (int i = 0; i < 2; ++i) { l.hi[i] = take(x); l.lo[i] = take(x); }
    l.a = take(q);
    l.p = take(q);
    auto parts_of = [&](int64_t batch) {
        const Form f = choose_form(l.sq, l.sq, rows < cols ? cols : rows, batch, true);
        return f.splits > 1 ? 4ull * (uint64_t)(f.splits * batch * l.sq * l.sq_ld) : 0ull;
    };
    const int64_t tail = n % l.group;            // the last group, where it is not full, may take more splits
    const uint64_t parts = std::max(parts_of(l.group), tail ? parts_of(tail) : 0ull);
    l.parts = take(parts);
    l.total = at;
    return l;
}

// The tensor maps of a call, made once: its arrays stay where they are from step to step.  X and its two words exist twice, in
// turn.
struct Maps {
    CUtensorMap x_k[2], x_k_narrow[2];            // X (hi) as a K-major operand (k = columns) of 128 or 64 rows per CTA
    CUtensorMap x_mn[2];                          // ... as an MN-major one (k = rows); its boxes are 64 wide either way
    CUtensorMap x_hi[2], x_lo[2];                 // X in chunks of 32 rows x 64 columns
    CUtensorMap a_op, a_op_narrow, p_op, p_op_narrow;      // the squares as K-major operands
    CUtensorMap a_chunk, a_mirror, p_chunk, p_mirror;      // ... as chunks, and as the mirrored ones (64 rows x 32 columns)
};

int make_maps(Maps* m, uint16_t* const* hi, uint16_t* const* lo, const uint16_t* a, const uint16_t* p, int64_t rows, int64_t cols, int64_t batch, const Layout& l)
{
    const int64_t xs = rows * l.ld, ps = l.sq * l.sq_ld;
    int rc = CAST_OK;
    auto also = [&rc](int r) { if (rc == CAST_OK) rc = r; };
    for (int i = 0; i < 2; ++i) {
        also(operand_map<false>(&m->x_k[i], hi[i], rows, cols, batch, l.ld, xs, 128));
        also(operand_map<false>(&m->x_k_narrow[i], hi[i], rows, cols, batch, l.ld, xs, 64));
        also(operand_map<true>(&m->x_mn[i], hi[i], cols, rows, batch, l.ld, xs, 128));
        also(make_map(&m->x_hi[i], hi[i], 2, cols, rows, batch, l.ld, xs, 64, 32, true));
        also(make_map(&m->x_lo[i], lo[i], 2, cols, rows, batch, l.ld, xs, 64, 32, true));
    }
    auto square = [&](const uint16_t* x, CUtensorMap* op, CUtensorMap* narrow, CUtensorMap* chunk, CUtensorMap* mirror) {
        also(operand_map<false>(op, x, l.sq, l.sq, batch, l.sq_ld, ps, 128));
        also(operand_map<false>(narrow, x, l.sq, l.sq, batch, l.sq_ld, ps, 64));
        also(make_map(chunk, x, 2, l.sq, l.sq, batch, l.sq_ld, ps, 64, 32, true));
        also(make_map(mirror, x, 2, l.sq, l.sq, batch, l.sq_ld, ps, 32, 64, false));
    };
    square(a, &m->a_op, &m->a_op_narrow, &m->a_chunk, &m->a_mirror);
    square(p, &m->p_op, &m->p_op_narrow, &m->p_chunk, &m->p_mirror);
    return rc;
}

// A = down X X^T over the batch (`cur`: which X), the tall form from X^T; then P = c A A + b A + a I.
template <int CG, int BN, bool MN>
int gram_product(const Maps& m, int cur, int64_t mn, int64_t k, int64_t batch, float down, const float* gain, cudaStream_t stream)
{
    Shape s;
    SymEpi<false> epi;
    int rc;
    if ((rc = make_shape<CG, BN, MN, MN, SymEpi<false>>(&s, false, mn, mn, k, batch, 1, 1)) != CAST_OK) return rc;
    epi.map_out = epi.map_aux = m.a_chunk;
    epi.map_mirror = m.a_mirror;
    epi.gain = gain;
    epi.traces = nullptr;
    epi.scale = down;
    epi.add = epi.diag = 0.0f;
    const bool narrow = BN / CG == 64;
    return launch<CG, BN, MN, MN>(MN ? m.x_mn[cur] : m.x_k[cur], MN ? m.x_mn[cur] : narrow ? m.x_k_narrow[cur] : m.x_k[cur],
                                  s, epi, stream);
}

template <int CG, int BN>
int poly_product(const Maps& m, int64_t mn, int64_t batch, const float* q, float* traces, cudaStream_t stream)
{
    Shape s;
    SymEpi<true> epi;
    int rc;
    if ((rc = make_shape<CG, BN, false, false, SymEpi<true>>(&s, false, mn, mn, mn, batch, 1, 1)) != CAST_OK) return rc;
    epi.map_out = m.p_chunk;
    epi.map_mirror = m.p_mirror;
    epi.map_aux = m.a_chunk;
    epi.gain = nullptr;
    epi.traces = traces;
    epi.diag = q[0];
    epi.add = q[1];
    epi.scale = q[2];
    return launch<CG, BN, false, false>(m.a_op, BN / CG == 64 ? m.a_op_narrow : m.a_op, s, epi, stream);
}

// A in splits of k: their sums, then the kernel that adds them.
template <int CG, int BN, bool MN>
int gram_parts(int splits, const Maps& m, int cur, int64_t mn, int64_t k, int64_t batch, float down, const float* gain, float* parts, uint16_t* a, int64_t ld,
               cudaStream_t stream)
{
    Shape s;
    PartEpi epi;
    int rc;
    if ((rc = make_shape<CG, BN, MN, MN, PartEpi>(&s, false, mn, mn, k, batch, splits, 1)) != CAST_OK) return rc;
    if ((rc = make_map(&epi.map_out, parts, 4, mn, mn, batch * s.splits, ld, mn * ld, 32, 32, true)) != CAST_OK) return rc;
    const bool narrow = BN / CG == 64;
    if ((rc = launch<CG, BN, MN, MN>(MN ? m.x_mn[cur] : m.x_k[cur], MN ? m.x_mn[cur] : narrow ? m.x_k_narrow[cur] : m.x_k[cur], s, epi, stream)) != CAST_OK) return rc;
    const int64_t blocks = (mn + 31) / 32;
    return launch_chained(false, add_parts_kernel, dim3((unsigned)(blocks * (blocks + 1) / 2), (unsigned)batch), 256, 0, stream, 1, parts, a, gain, s.splits,
                          (int)mn, ld, ld, down);
}

template <bool MN>
int gram_product(const Form& form, const Maps& m, int cur, int64_t mn, int64_t k, int64_t batch, float down, const float* gain, float* parts, uint16_t* a,
                 int64_t ld, cudaStream_t stream)
{
    const TileForm f = form.tile;
    if (form.splits > 1) {
        if (f == kPair256) return gram_parts<2, 256, MN>(form.splits, m, cur, mn, k, batch, down, gain, parts, a, ld, stream);
        if (f == kSingle128) return gram_parts<1, 128, MN>(form.splits, m, cur, mn, k, batch, down, gain, parts, a, ld, stream);
        return gram_parts<1, 64, MN>(form.splits, m, cur, mn, k, batch, down, gain, parts, a, ld, stream);
    }
    if (f == kPair256) return gram_product<2, 256, MN>(m, cur, mn, k, batch, down, gain, stream);
    if (f == kSingle128) return gram_product<1, 128, MN>(m, cur, mn, k, batch, down, gain, stream);
    return gram_product<1, 64, MN>(m, cur, mn, k, batch, down, gain, stream);
}

int poly_product(TileForm f, const Maps& m, int64_t mn, int64_t batch, const float* q, float* traces, cudaStream_t stream)
{
    if (f == kPair256) return poly_product<2, 256>(m, mn, batch, q, traces, stream);
    if (f == kSingle128) return poly_product<1, 128>(m, mn, batch, q, traces, stream);
    return poly_product<1, 64>(m, mn, batch, q, traces, stream);
}

struct StepCall {
    const Maps* maps;
    const OutTable* out;
    const float* gain;
    const float* traces;
    int64_t rows, cols, batch, sq;
    float scale;
    int cur;                          // which X
    bool lo_in, lo_out, last, vec;
    cudaStream_t stream;
};

// X' = P X (wide) or X P (tall)
template <int CG, int BN, bool WIDE, class Epi>
int step_product(const StepCall& c, Epi& epi)
{
    Shape s;
    int rc;
    const Maps& m = *c.maps;
    const bool narrow = BN / CG == 64;
    if ((rc = make_shape<CG, BN, false, WIDE, Epi>(&s, false, c.rows, c.cols, c.sq, c.batch, 1, 16 / CG)) != CAST_OK) return rc;
    if (WIDE) return launch<CG, BN, false, WIDE>(m.p_op, m.x_mn[c.cur], s, epi, c.stream);
    return launch<CG, BN, false, WIDE>(m.x_k[c.cur], narrow ? m.p_op_narrow : m.p_op, s, epi, c.stream);
}

template <int CG, int BN, bool WIDE, bool LO_IN, bool LO_OUT>
int next_product(const StepCall& c)
{
    const Maps& m = *c.maps;
    StepEpi<LO_IN, LO_OUT> epi;
    epi.map_hi = m.x_hi[c.cur ^ 1];
    epi.map_lo = m.x_lo[c.cur ^ 1];
    epi.map_lo_in = m.x_lo[c.cur];
    epi.gain = c.gain;
    epi.traces = c.traces;
    epi.sq = (int)c.sq;
    return step_product<CG, BN, WIDE>(c, epi);
}

template <int CG, int BN, bool WIDE, bool LO_IN>
int result_product(const StepCall& c)
{
    ResultEpi<LO_IN> epi;
    epi.map_lo_in = c.maps->x_lo[c.cur];
    epi.out = *c.out;
    epi.gain = c.gain;
    epi.traces = c.traces;
    epi.sq = (int)c.sq;
    epi.scale = c.scale;
    epi.vec = c.vec;
    return step_product<CG, BN, WIDE>(c, epi);
}

template <int CG, int BN, bool WIDE>
int any_product(const StepCall& c)
{
    if (c.last) return c.lo_in ? result_product<CG, BN, WIDE, true>(c) : result_product<CG, BN, WIDE, false>(c);
    if (c.lo_in) return c.lo_out ? next_product<CG, BN, WIDE, true, true>(c) : next_product<CG, BN, WIDE, true, false>(c);
    return c.lo_out ? next_product<CG, BN, WIDE, false, true>(c) : next_product<CG, BN, WIDE, false, false>(c);
}

template <bool WIDE>
int step_product(TileForm f, const StepCall& c)
{
    if (f == kPair256) return any_product<2, 256, WIDE>(c);
    if (f == kSingle128) return any_product<1, 128, WIDE>(c);
    return any_product<1, 64, WIDE>(c);
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
                          reinterpret_cast<uint16_t*>(ws + l.hi[0]), reinterpret_cast<uint16_t*>(ws + l.lo[0]), reinterpret_cast<float*>(ws + l.gains), units, (uint32_t)(cols / VEC), l.ld,
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
    int rc;
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
        OutTable to;
        bool in_vec = cols % 8 == 0, out_vec = cols % 8 == 0;
        for (int64_t i = 0; i < batch; ++i) {
            in.p[i] = updates[first + i];
            to.p[i] = out[first + i];
            in_vec = in_vec && !((uintptr_t)in.p[i] & 15u);
            out_vec = out_vec && !((uintptr_t)to.p[i] & 15u);
        }
        for (int64_t i = batch; i < kGroup; ++i) { in.p[i] = nullptr; to.p[i] = nullptr; }
        if (updates_bf16) rc = in_vec ? launch_first<true, 8>(first == 0, in, batch, rows, cols, ws, l, eps, st) : launch_first<true, 1>(first == 0, in, batch, rows, cols, ws, l, eps, st);
        else rc = in_vec ? launch_first<false, 8>(first == 0, in, batch, rows, cols, ws, l, eps, st) : launch_first<false, 1>(first == 0, in, batch, rows, cols, ws, l, eps, st);
        if (rc != CAST_OK) return rc;
        const Form gram = choose_form(l.sq, l.sq, big, batch, true);
        const TileForm poly = choose_form(l.sq, l.sq, l.sq, batch, true, 1).tile, step = choose_form(rows, cols, l.sq, batch, false, 1).tile;
        float* parts = reinterpret_cast<float*>(ws + l.parts);
        float* traces = reinterpret_cast<float*>(ws + l.traces);
        Maps maps;
        if ((rc = make_maps(&maps, hi, lo, a, p, rows, cols, batch, l)) != CAST_OK) return rc;
        bool has_lo = !updates_bf16;
        for (int k = 0; k < steps; ++k) {
            const float* q = coeffs ? coeffs + 3 * k : kQuintic;
            const int cur = k & 1;
            const float* gain = updates_bf16 && k == 0 ? reinterpret_cast<const float*>(ws + l.gains) : nullptr;
            rc = wide ? gram_product<false>(gram, maps, cur, l.sq, big, batch, 1.0f / (kX * kX), gain, parts, a, l.sq_ld, st)
                      : gram_product<true>(gram, maps, cur, l.sq, big, batch, 1.0f / (kX * kX), gain, parts, a, l.sq_ld, st);
            if (rc != CAST_OK) return rc;
            if ((rc = poly_product(poly, maps, l.sq, batch, q, traces, st)) != CAST_OK) return rc;
            const bool last = k + 1 == steps;
            float amplify = 1.0f;      // of a small direction of X', by the steps after this one
            for (int j = k + 1; j < steps; ++j) amplify *= std::fabs(coeffs ? coeffs[3 * j] : kQuintic[0]);
            const bool lo_out = !last && amplify > kAmplify;
            const StepCall c = {&maps, &to, gain, traces, rows, cols, batch, l.sq, scale / kX, cur, has_lo, lo_out, last, out_vec, st};
            if ((rc = wide ? step_product<true>(step, c) : step_product<false>(step, c)) != CAST_OK) return rc;
            has_lo = lo_out;
        }
    }
    return CAST_OK;
}
