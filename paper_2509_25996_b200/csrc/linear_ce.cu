// Softmax cross entropy of a linear head, l = hidden weight^T, and its gradients.  The logits are not stored; for the gradients their
// exponentials are, in bf16, a piece of the tokens at a time (below).
//
// With r_i = h_i . w_label(i) (the target logit) and S_i = sum_{j != label} e^(l_ij - r_i):
//     loss_i = log(1 + S_i),   p_ij = e^(l_ij - r_i) / (1 + S_i),   1 - p_i,label = S_i / (1 + S_i)
// so nothing cancels for a confident token, and a tile of logits needs no statistics of the rest of its row: the product's
// epilogue turns the accumulators into E_ij = e^(l_ij - r_i) (0 at the label) and its row sums at once.  Per piece of tokens:
//     target logits   r_i, one warp per token
//     E = exp(H W^T - r)            product, epilogue writes E (bf16) and the row sums of half a tile each
//     finish          S, loss, a_i = s / (1 + S_i), b_i = s S_i / (1 + S_i), and a H as bf16
//     B_v = sum_{label = v} b H     fp32 rows by label (the embedding gradient's sums), before the last piece's dW
//     dH = a (E W) - b W_label      product over the vocabulary; the label's row is added in fp32 by the epilogue
//     dW = E^T (a H) - B            product over the tokens; B is subtracted in fp32 by the epilogue
// The two backward products read E as it was written: no pass over it to apply the normaliser.
//
// E takes 2 bytes per logit of a piece, as much as logits in bf16 would: all of them, 262 MB, for 4096 tokens x 32000; pieces of
// 1 GiB bound it for more.  Several pieces accumulate dW in fp32 (2.1 GB for 128256 x 4096).  The loss alone needs neither.
// Range: e^(l - r) beyond e^40 (a target that is that improbable) would leave the range of the later sums.  The epilogue
// sees it in its row sum, forms that row's part of the tile relative to the tile's own maximum instead and says so by a negative
// sum; finish then brings the row to one reference.
//
// Rounding: the products take bf16 operands, so E and a H are rounded to bf16 (2^-8 relative at most); everything that is
// summed, and all statistics, are fp32.  The label's terms, the largest of a row, are never rounded before the result is: the two
// parts of a frequent label's row of dW nearly cancel where the head is calibrated and the hidden states have a common mean, so
// that a rounding of one of them would be 30 of the result's (measured: 5.3e-2 of such a row instead of 1.7e-3).
//
// Bounded by the tensor cores, for large calls at the clock that the power limit leaves them (1.3-1.4 GHz): 4096 tokens x 32000
// x 4096 2.51-2.59 ms (1260 TFLOP/s), 8192 x 128256 x 4096 20.2-20.8 ms (1260), loss alone of 2047 x 32000 x 5120 0.505 ms (1330).
// 1000 x 50257 x 768 takes 237 us (976): its three products (61, 56 and 58 us alone, tensor pipe 76-83 % busy) read 620 MB of
// operands each through L2; by a launch list they are 85 % of the call, target logits, finish, the join of dH and the label sums
// the rest.  48 x 32000 x 768 takes 59 us, where reading and writing the head once takes 15: seven launches in a chain, of which E
// and dW (49 MB of the head read, as many of its gradient written) are a quarter each, dH and its join a third.
#include <cmath>

#include "embed.cuh"
#include "tile_product.cuh"

namespace cast {
namespace {

using namespace product;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMostSum = 2.35e17f;        // e^40
constexpr int kHalves = 2;                  // a tile's columns are summed by two warps

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// A target logit as a power of two, kept finite (NaN stays), so that a target of no probability at all (a masked row of the head)
// leaves the other probabilities as they are: a difference with it must not be inf - inf.
constexpr float kFar = 3.0e38f;
__device__ __forceinline__ float base2(float ref)
{
    const float r = __fmul_rn(ref, kLog2e);          // rounded, whatever it is subtracted from
    return r < -kFar ? -kFar : r > kFar ? kFar : r;
}

// ------------------------------------------------------------------------------------------------ target logits

// refs[t] = h_t . w_label, 0 without a label.  One warp per token; dim % 8 == 0.  For dW's label terms, the CTAs after the tokens' own
// begin the order of the labels, and those after them (from `fill0` on) write -1 to `row_of`, the row in B of every label.
__global__ void __launch_bounds__(kRankThreads)
target_logit_kernel(const uint16_t* __restrict__ hidden, const uint16_t* __restrict__ weight, const int32_t* __restrict__ labels,
                    float* __restrict__ refs, int64_t tokens, int vocab, int dim, unsigned own, unsigned fill0, const SortStart start,
                    int4* __restrict__ row_of)
{
    chain_next();
    if (blockIdx.x >= fill0) {
        const int64_t v = (int64_t)(blockIdx.x - fill0) * kRankThreads + threadIdx.x;
        if (4 * v < vocab) row_of[v] = make_int4(-1, -1, -1, -1);        // padded to whole vectors
        return;
    }
    if (blockIdx.x >= own) {
        rank_keys(labels, start, tokens, (uint32_t)vocab, blockIdx.x - own, fill0 - own);
        return;
    }
    const int64_t t = (int64_t)blockIdx.x * (kRankThreads / 32) + (threadIdx.x >> 5);
    if (t >= tokens) return;
    const int lane = (int)threadIdx.x & 31;
    const int label = labels[t];
    float sum = 0.0f;
    if ((unsigned)label < (unsigned)vocab) {
        const uint4* h = reinterpret_cast<const uint4*>(hidden + t * dim);
        const uint4* w = reinterpret_cast<const uint4*>(weight + (int64_t)label * dim);
        // four vectors of each row at a time, the last ones too: a loop's remainder would wait for one load after the other
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int i0 = lane; i0 < dim / 8; i0 += 128) {
            uint4 a[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = i0 + 32 * j < dim / 8;
                a[j] = in ? __ldg(h + i0 + 32 * j) : zero;
                b[j] = in ? __ldg(w + i0 + 32 * j) : zero;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum += lo16(a[j].x) * lo16(b[j].x) + hi16(a[j].x) * hi16(b[j].x) + lo16(a[j].y) * lo16(b[j].y) + hi16(a[j].y) * hi16(b[j].y) +
                       lo16(a[j].z) * lo16(b[j].z) + hi16(a[j].z) * hi16(b[j].z) + lo16(a[j].w) * lo16(b[j].w) + hi16(a[j].w) * hi16(b[j].w);
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (lane == 0) refs[t] = sum;
}

// ------------------------------------------------------------------------------------------------ E and its row sums

struct ExpEpi : StoringEpi {
    static constexpr bool kInputsOnly = true;
    // 1024 k: a logit of typical operands loses 1e-6 of itself whatever k is.  Loss of 2047 tokens x 32000 x 5120 against 64 bits:
    // 3.0e-7 (in one run 1.7e-6), 509 us (507); with 16384 columns 7.4e-7 (1.4e-5).
    static constexpr int kRunStages = 16;
    CUtensorMap map_e;
    const float* refs;           // target logits of the piece
    const int32_t* labels;
    float* sums;                 // [2 per tile: its halves][tokens]; negative: relative to `tops`
    float* tops;                 // likewise, base 2
    int write_e;

    // One pass over the accumulator row relative to ref2: returns the sum; writes E.
    template <int BN>
    __device__ __forceinline__ float pass(const Shape& s, EpiTile& e, float ref2, int label, bool active) const
    {
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll 1
        for (int c = e.c0; c < e.c1; c += 64) {
            const int n = e.col0 + c;
            if (n >= s.n) break;
            uint32_t slot = 0;
            if (write_e) slot = slot_acquire(e);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
                const int n1 = n + 32 * h;
                const bool special = !active || (unsigned)(label - n1) < 32u || n1 + 32 > s.n;
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = ex2(fmaf(v[i], kLog2e, -ref2));
                if (__any_sync(0xFFFFFFFFu, special)) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!active || n1 + i == label || n1 + i >= s.n) v[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 32; i += 2) { s0 += v[i]; s1 += v[i + 1]; }
                if (write_e) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        slot_write(slot, e.lane, 4 * h + q, pack2(v[8 * q], v[8 * q + 1]), pack2(v[8 * q + 2], v[8 * q + 3]),
                                   pack2(v[8 * q + 4], v[8 * q + 5]), pack2(v[8 * q + 6], v[8 * q + 7]));
                }
            }
            if (write_e) slot_store(e, slot, &map_e, n, e.row0, 0, e.row0 < s.m);
        }
        return s0 + s1;
    }

    __device__ __forceinline__ void prefetch() const { if (write_e) prefetch_map(&map_e); }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State&) const
    {
        const int row = e.row0 + e.lane;
        int label = -1;
        float ref2 = 0.0f;
        if (row < s.m) {
            label = __ldg(labels + row);
            if ((unsigned)label >= (unsigned)s.n) label = -1;
            ref2 = base2(__ldg(refs + row));
        }
        const int64_t at = (int64_t)(e.tile.tn * kHalves + (e.c0 ? 1 : 0)) * s.m;
        const bool active = label >= 0;
        float sum = pass<BN>(s, e, ref2, label, active);
        const bool over = !(sum <= kMostSum);          // also a sum that is not a number
        if (__any_sync(0xFFFFFFFFu, over)) {
            float top = -INFINITY;
#pragma unroll 1
            for (int c = e.c0; c < e.c1; c += 32) {
                float v[32];
                if (e.col0 + c >= s.n) break;
                tmem_load32(e.acc + (uint32_t)c, v);
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (e.col0 + c + i != label && e.col0 + c + i < s.n) top = fmaxf(top, v[i]);
            }
            const float top2 = top * kLog2e;
            if (e.lane == 0) store_wait_all();          // the first pass has been written before the second overwrites it
            __syncwarp();
            const float again = pass<BN>(s, e, over ? top2 : ref2, label, active);
            if (over) {
                sum = -again;
                tops[at + row] = top2;
            }
        }
        if (row < s.m) sums[at + row] = sum;
        return true;
    }
};

// ------------------------------------------------------------------------------------------------ finish

constexpr int kFinishTokens = 8;      // 8 tokens x 4 bytes: one sector of a row of `sums`

struct FinishArgs {
    const uint16_t* hidden;
    const int32_t* labels;
    const float* refs;
    const float* sums;
    const float* tops;
    float* loss;
    float* a;                 // s / (1 + S), 0 without a label
    float* b;                 // s S / (1 + S)
    uint16_t* e;              // [tokens][e_ld] or nullptr
    uint16_t* scaled;         // a H, bf16, or nullptr
    int64_t tokens, e_ld;
    int vocab, dim, n_tiles, tile_cols;
    float grad_scale;
};

constexpr int kAhead = 4;             // vectors of the token's hidden row that a lane loads before it needs them

__global__ void __launch_bounds__(256)
finish_kernel(const __grid_constant__ FinishArgs p)
{
    __shared__ float part[32][kFinishTokens];
    __shared__ float sh_a[kFinishTokens], sh_ref[kFinishTokens];
    __shared__ int sh_over[kFinishTokens];
    chain_next();
    const int warp = (int)threadIdx.x >> 5, wl = (int)threadIdx.x & 31;      // later: one warp per token
    const int64_t t0 = (int64_t)blockIdx.x * kFinishTokens;
    const uint4* h = reinterpret_cast<const uint4*>(p.hidden + (t0 + warp) * p.dim);
    uint4 ahead[kAhead];
    if (p.scaled && t0 + warp < p.tokens) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (wl + 32 * i < p.dim / 8) ahead[i] = __ldg(h + wl + 32 * i);
    }
    chain_wait();
    const int k = (int)threadIdx.x & 7, lane = (int)threadIdx.x >> 3;
    const int64_t t = (int64_t)blockIdx.x * kFinishTokens + k;
    const bool in = t < p.tokens;
    const int label = in ? p.labels[t] : -1;
    const bool active = (unsigned)label < (unsigned)p.vocab;
    const float ref = in ? p.refs[t] : 0.0f, ref2 = base2(ref);

    // largest reference of the row's tiles (the target logit where none was too large)
    float top2 = ref2;
    bool over = false;
    float sum = 0.0f;
    if (active) {
        for (int i0 = lane; i0 < p.n_tiles; i0 += 256) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i0 + 32 * j < p.n_tiles ? p.sums[(int64_t)(i0 + 32 * j) * p.tokens + t] : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                over |= !(v[j] >= 0.0f);
                sum += v[j];
            }
        }
    }
    if (__syncthreads_or(over)) {           // rare: bring the tiles of such rows to one reference
        if (over)
            for (int i = lane; i < p.n_tiles; i += 32)
                if (!(p.sums[(int64_t)i * p.tokens + t] >= 0.0f)) top2 = fmaxf(top2, p.tops[(int64_t)i * p.tokens + t]);
        part[lane][k] = top2;
        __syncthreads();
        for (int i = 0; i < 32; ++i) top2 = fmaxf(top2, part[i][k]);
        __syncthreads();
        sum = 0.0f;
        if (active)
            for (int i = lane; i < p.n_tiles; i += 32) {
                const float v = p.sums[(int64_t)i * p.tokens + t];
                sum += v >= 0.0f ? v * ex2(ref2 - top2) : -v * ex2(p.tops[(int64_t)i * p.tokens + t] - top2);
            }
    }
    part[lane][k] = sum;
    __syncthreads();
    if (threadIdx.x < kFinishTokens) {
        float s = 0.0f;
        for (int i = 0; i < 32; ++i) s += part[i][k];
        // the epilogue subtracted ref log2(e) rounded to fp32, the same for the whole row: put the rest of that product back
        const float missed = top2 == ref2 && fabsf(ref2) < kFar ? fmaf(ref, kLog2e, -ref2) * kLn2 : 0.0f;
        if (ref == INFINITY) s = NAN;          // as is a row with any other infinite logit
        float loss = 0.0f, a = 0.0f, b = 0.0f;
        if (active) {
            const float own = ex2(ref2 - top2);          // the target's own term, 1 unless the reference moved
            if (top2 == ref2) {
                s -= s * missed;
                loss = log1pf(s);
            } else {
                loss = (top2 * kLn2 - ref) + logf(own + s);
            }
            a = (p.grad_scale - p.grad_scale * missed) / (own + s);
            b = p.grad_scale * (s / (own + s));
        }
        if (in) {
            p.loss[t] = loss;
            if (p.a) { p.a[t] = a; p.b[t] = b; }
        }
        sh_a[k] = a;
        sh_ref[k] = top2;
        sh_over[k] = active && top2 != ref2;
    }
    __syncthreads();
    if (t0 + warp >= p.tokens) return;
    if (p.scaled) {
        const float a = sh_a[warp];
        uint4* o = reinterpret_cast<uint4*>(p.scaled + (t0 + warp) * p.dim);
        auto scaled = [a](const uint4& x) {
            if (a == 0.0f) return make_uint4(0u, 0u, 0u, 0u);        // a token without a label contributes nothing, whatever it holds
            return make_uint4(pack2(a * lo16(x.x), a * hi16(x.x)), pack2(a * lo16(x.y), a * hi16(x.y)),
                              pack2(a * lo16(x.z), a * hi16(x.z)), pack2(a * lo16(x.w), a * hi16(x.w)));
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (wl + 32 * i < p.dim / 8) o[wl + 32 * i] = scaled(ahead[i]);
        for (int i0 = wl + 32 * kAhead; i0 < p.dim / 8; i0 += 32 * kAhead) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (i0 + 32 * i < p.dim / 8) ahead[i] = __ldg(h + i0 + 32 * i);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (i0 + 32 * i < p.dim / 8) o[i0 + 32 * i] = scaled(ahead[i]);
        }
    }
    if (p.e && sh_over[warp]) {
        uint16_t* row = p.e + (t0 + warp) * p.e_ld;
        const float r2 = base2(p.refs[t0 + warp]);
        for (int j = wl; j < p.vocab; j += 32) {
            const int64_t at = (int64_t)(j / p.tile_cols) * p.tokens + t0 + warp;
            const float from = p.sums[at] >= 0.0f ? r2 : p.tops[at];
            row[j] = (uint16_t)(pack2(__uint_as_float((uint32_t)row[j] << 16) * ex2(from - sh_ref[warp]), 0.0f) & 0xFFFFu);
        }
    }
}

// ------------------------------------------------------------------------------------------------ gradients

__device__ __forceinline__ void store_bf16_row(uint32_t slot, int lane, int half, const float (&v)[32])
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        slot_write(slot, lane, 4 * half + q, pack2(v[8 * q], v[8 * q + 1]), pack2(v[8 * q + 2], v[8 * q + 3]),
                   pack2(v[8 * q + 4], v[8 * q + 5]), pack2(v[8 * q + 6], v[8 * q + 7]));
}

// One fp32 slot holds 32 columns.
__device__ __forceinline__ void store_f32_row(uint32_t slot, int lane, const float (&v)[32])
{
#pragma unroll
    for (int q = 0; q < 8; ++q)
        slot_write(slot, lane, q, __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
}

// dH tile: a (E W) - b W_label as bf16, or with several splits over the vocabulary the plain sums as fp32.
struct HiddenGradEpi : StoringEpi {
    CUtensorMap map_out;         // bf16 [tokens][dim], or fp32 [splits][tokens][dim]
    const float* a;
    const float* b;
    const int32_t* labels;
    const uint16_t* weight;
    int vocab, partial;

    __device__ __forceinline__ void prefetch() const { prefetch_map(&map_out); }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State&) const
    {
        if (partial) {
#pragma unroll 1
            for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 32) {
                float v[32];
                const uint32_t slot = slot_acquire(e);
                tmem_load32(e.acc + (uint32_t)c, v);
                store_f32_row(slot, e.lane, v);
                slot_store(e, slot, &map_out, e.col0 + c, e.row0, e.tile.split, e.row0 < s.m);
            }
            return true;
        }
        const int row = e.row0 + e.lane;
        float fa = 0.0f, fb = 0.0f;
        int label = -1;
        if (row < s.m) {
            label = __ldg(labels + row);
            if ((unsigned)label >= (unsigned)vocab) label = -1;
            fa = __ldg(a + row);
            fb = __ldg(b + row);
        }
        const uint16_t* w = weight + (int64_t)(label < 0 ? 0 : label) * s.n;
#pragma unroll 1
        for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 64) {
            const uint32_t slot = slot_acquire(e);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int n1 = e.col0 + c + 32 * h;
                uint4 x[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)        // dim % 8 == 0: whole vectors
                    x[q] = (label >= 0 && n1 + 8 * q < s.n) ? __ldg(reinterpret_cast<const uint4*>(w + n1) + q) : make_uint4(0u, 0u, 0u, 0u);
                float v[32];
                tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t u[4] = {x[q].x, x[q].y, x[q].z, x[q].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float& lo = v[8 * q + 2 * i];
                        float& hi = v[8 * q + 2 * i + 1];
                        lo = label >= 0 ? fa * lo - fb * lo16(u[i]) : 0.0f;
                        hi = label >= 0 ? fa * hi - fb * hi16(u[i]) : 0.0f;
                    }
                }
                store_bf16_row(slot, e.lane, h, v);
            }
            slot_store(e, slot, &map_out, e.col0 + c, e.row0, 0, e.row0 < s.m);
        }
        return true;
    }
};

// Adds the splits' sums in order and finishes dH.  One thread per 8 columns.
constexpr int kJoinThreads = 64;

__global__ void __launch_bounds__(kJoinThreads)
join_hidden_grad_kernel(const float* __restrict__ partial, const float* __restrict__ a, const float* __restrict__ b,
                        const int32_t* __restrict__ labels, const uint16_t* __restrict__ weight, uint16_t* __restrict__ out,
                        int64_t tokens, int dim, int vocab, int splits)
{
    chain_next();
    const int64_t u = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    const int per = dim / 8;
    if (u >= tokens * per) return;
    const int64_t t = u / per;
    const int c = (int)(u - t * per) * 8;
    const int label = __ldg(labels + t);
    const bool active = (unsigned)label < (unsigned)vocab;
    uint4 w = make_uint4(0u, 0u, 0u, 0u), r = w;
    if (active) w = __ldg(reinterpret_cast<const uint4*>(weight + (int64_t)label * dim + c));
    chain_wait();
    if (active) {
        float v[8] = {};
        const float4* p = reinterpret_cast<const float4*>(partial + t * dim + c);
        const int64_t step = tokens * dim / 4;
        const float fa = a[t], fb = b[t];
        for (int s0 = 0; s0 < splits; s0 += 8, p += 8 * step) {
            float4 x[8], y[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const bool in = s0 + s < splits;
                x[s] = in ? __ldg(p + s * step) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                y[s] = in ? __ldg(p + s * step + 1) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                v[0] += x[s].x; v[1] += x[s].y; v[2] += x[s].z; v[3] += x[s].w;
                v[4] += y[s].x; v[5] += y[s].y; v[6] += y[s].z; v[7] += y[s].w;
            }
        }
        r = make_uint4(pack2(fa * v[0] - fb * lo16(w.x), fa * v[1] - fb * hi16(w.x)), pack2(fa * v[2] - fb * lo16(w.y), fa * v[3] - fb * hi16(w.y)),
                       pack2(fa * v[4] - fb * lo16(w.z), fa * v[5] - fb * hi16(w.z)), pack2(fa * v[6] - fb * lo16(w.w), fa * v[7] - fb * hi16(w.w)));
    }
    *reinterpret_cast<uint4*>(out + t * dim + c) = r;
}

// dW tile: bf16 result after the last piece, less the label's rows; fp32 running sums before it.
struct WeightGradEpi : StoringEpi {
    CUtensorMap map_out;         // bf16 [vocab][dim]
    CUtensorMap map_acc;         // fp32 [vocab][dim]
    const float* acc;
    const float* rows;           // B, and the row of it that belongs to a label
    const int32_t* row_of;
    int add, last;

    __device__ __forceinline__ void add_running(const Shape& s, int row, int n1, float (&v)[32]) const
    {
        if (row >= s.m) return;
        const float* p = acc + (int64_t)row * s.n + n1;
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (n1 + 4 * q < s.n) {
                const float4 x = __ldcs(reinterpret_cast<const float4*>(p) + q);
                v[4 * q] += x.x; v[4 * q + 1] += x.y; v[4 * q + 2] += x.z; v[4 * q + 3] += x.w;
            }
    }

    __device__ __forceinline__ void prefetch() const { prefetch_map(last ? &map_out : &map_acc); }

    template <int BM, int BN>
    __device__ __forceinline__ bool tile(const Shape& s, EpiTile& e, State&) const
    {
        const int row = e.row0 + e.lane;
        if (last) {
            const int own = row < s.m ? __ldg(row_of + row) : -1;
            const float* b = rows + (int64_t)(own < 0 ? 0 : own) * s.n;
            // most tiles of a short call have none (without the branch 48 tokens x 32000 x 768 take 2 us longer)
            const bool labels = __any_sync(0xFFFFFFFFu, own >= 0);
#pragma unroll 1
            for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 64) {
                const uint32_t slot = slot_acquire(e);
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    const int n1 = e.col0 + c + 32 * h;
                    float v[32];
                    tmem_load32(e.acc + (uint32_t)(c + 32 * h), v);
                    if (add) add_running(s, row, n1, v);
                    if (labels) {
                        float4 x[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            x[q] = own >= 0 && n1 + 4 * q < s.n ? __ldg(reinterpret_cast<const float4*>(b + n1) + q) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            v[4 * q] -= x[q].x; v[4 * q + 1] -= x[q].y; v[4 * q + 2] -= x[q].z; v[4 * q + 3] -= x[q].w;
                        }
                    }
                    store_bf16_row(slot, e.lane, h, v);
                }
                slot_store(e, slot, &map_out, e.col0 + c, e.row0, 0, e.row0 < s.m);
            }
        } else {
#pragma unroll 1
            for (int c = e.c0; c < e.c1 && e.col0 + c < s.n; c += 32) {
                const uint32_t slot = slot_acquire(e);
                float v[32];
                tmem_load32(e.acc + (uint32_t)c, v);
                if (add) add_running(s, row, e.col0 + c, v);
                store_f32_row(slot, e.lane, v);
                slot_store(e, slot, &map_acc, e.col0 + c, e.row0, 0, e.row0 < s.m);
            }
        }
        return true;
    }
};

// ------------------------------------------------------------------------------------------------ host

constexpr uint64_t kDefaultPieceBytes = 1ull << 30;       // of E

int64_t e_row_elems(int64_t vocab) { return (vocab + 63) / 64 * 64; }

int64_t piece_of(int64_t tokens, int64_t vocab, int64_t piece_tokens)
{
    if (piece_tokens > 0) return piece_tokens < tokens ? piece_tokens : tokens;
    int64_t fit = (int64_t)(kDefaultPieceBytes / (2ull * (uint64_t)e_row_elems(vocab)));
    if (fit < 256) fit = 256;
    if (fit >= tokens) return tokens;
    // equal pieces, whole tiles of tokens
    const int64_t n = (tokens + fit - 1) / fit;
    const int64_t each = (tokens + n - 1) / n;
    return (each + 255) / 256 * 256;
}

// Tiles of 256 x 256 on CTA pairs, or of 128 x 128 where a pair's second CTA would have no tokens.  Loss and both gradients,
// us on pairs / on single CTAs: 128 tokens x 32000 x 768 68 / 58, 64 x 32000 x 4096 185 / 171; 160 x 32000 x 4096 199 / 224,
// 256 x 128256 x 2048 420 / 462.
bool paired(int64_t tokens) { return tokens > 128; }
int64_t tile_cols(int64_t tokens) { return (paired(tokens) ? 256 : 128) / kHalves; }      // of one row sum

// Rows of `sums`: the halves of all tiles, the last one's empty half too.
int64_t sum_rows(int64_t vocab, int64_t tokens)
{
    const int64_t tile = tile_cols(tokens) * kHalves;
    return (vocab + tile - 1) / tile * kHalves;
}

// Splits of the vocabulary for dH: few tokens give few tiles, and each has the whole vocabulary to sum.  The time of
// `splits` is taken as rounds of tiles x (blocks + 8 for filling and draining the pipeline), in blocks (~0.3 us for a pair),
// plus writing and reading the partial sums at ~5 TB/s.  A split has to save a twentieth of that, which the model does not resolve,
// as its sums take memory.  Loss and dH, us, with that margin / without: 512 x 128256 x 4096 (2 splits / 9) 787 / 793, 57 x 11076 x
// 192 (29 / 44) 37 / 43, 430 x 59492 x 192 (31 / 36) 112 / 119, 814 x 95519 x 248 (17 / 18) 202 / 211, 2 x 45992 x 1112 (15 / 16) 94 / 96;
// 572 x 2176 x 1488 (1 / 3) 60 / 57, 55 x 1010 x 1800 (1 / 4) 43 / 42, 4096 x 32000 x 4096 (1 / 2) 1634 / 1621.
int hidden_splits(int64_t tokens, int64_t vocab, int64_t dim, int sms)
{
    const bool two = paired(tokens);
    const int64_t units = two ? sms / 2 : sms, bm = two ? 256 : 128, bn = two ? 256 : 128;
    const int64_t tiles = ((tokens + bm - 1) / bm) * ((dim + bn - 1) / bn), blocks = (vocab + kBK - 1) / kBK;
    int best = 1;
    int64_t best_cost = INT64_MAX;
    for (int s = 1; s <= 64 && s <= blocks; ++s) {
        const int64_t rounds = (tiles * s + units - 1) / units;
        const int64_t cost = rounds * ((blocks + s - 1) / s + 8) + (s > 1 ? 8 + s * tokens * dim * 8 / (two ? 1500000 : 1000000) : 0);
        if (cost + cost / 20 < best_cost) { best_cost = cost; best = s; }
    }
    return best;
}

struct Layout {
    int64_t piece, pieces, e_ld, n_tiles;
    int splits;
    uint64_t e, scaled, refs, a, b, sums, tops, partial, acc, scatter, rows, row_of, total;
};

int layout_of(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece_tokens, bool want_h, bool want_w, int sms, Layout* l)
{
    l->piece = piece_of(tokens, vocab, piece_tokens);
    l->pieces = (tokens + l->piece - 1) / l->piece;
    l->e_ld = e_row_elems(vocab);
    l->n_tiles = sum_rows(vocab, l->piece);
    // the last piece may be short enough for the narrower tiles
    const int64_t tail = tokens - (l->pieces - 1) * l->piece;
    const int64_t tail_tiles = sum_rows(vocab, tail);
    int s1 = 1, s2 = 1;
    if (want_h) { s1 = hidden_splits(l->piece, vocab, dim, sms); s2 = hidden_splits(tail, vocab, dim, sms); }
    l->splits = s1;
    const bool grads = want_h || want_w;
    uint64_t at = 0;
    auto take = [&at](uint64_t bytes) { const uint64_t o = at; at += align256(bytes); return o; };
    const uint64_t P = (uint64_t)l->piece, D = (uint64_t)dim;
    l->e = take(grads ? 2ull * P * (uint64_t)l->e_ld : 0);
    l->scaled = take(want_w ? 2ull * P * D : 0);
    l->refs = take(4ull * (uint64_t)tokens);
    l->a = take(grads ? 4ull * (uint64_t)tokens : 0);
    l->b = take(grads ? 4ull * (uint64_t)tokens : 0);
    const uint64_t stat = 4ull * (P * (uint64_t)l->n_tiles > (uint64_t)tail * (uint64_t)tail_tiles ? P * (uint64_t)l->n_tiles : (uint64_t)tail * (uint64_t)tail_tiles);
    l->sums = take(stat);
    l->tops = take(stat);
    const uint64_t p1 = s1 > 1 ? 4ull * (uint64_t)s1 * P * D : 0, p2 = s2 > 1 ? 4ull * (uint64_t)s2 * (uint64_t)tail * D : 0;
    l->partial = take(p1 > p2 ? p1 : p2);
    l->acc = take(want_w && l->pieces > 1 ? 4ull * (uint64_t)vocab * D : 0);
    l->scatter = take(want_w ? scatter_scratch_bytes(tokens, dim) : 0);
    l->rows = take(want_w ? 4ull * (uint64_t)compact_rows(tokens, vocab) * D : 0);
    l->row_of = take(want_w ? 4ull * (uint64_t)vocab : 0);
    l->total = at;
    return CAST_OK;
}

int check_ce_shape(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece_tokens)
{
    if (tokens < 1 || vocab < 1 || dim < 8 || dim % 8 != 0 || piece_tokens < 0) return CAST_ERR_SHAPE;
    if (tokens > 0x3FFFFFFF || vocab > 0x7FFFFF00 || dim > (1 << 20)) return CAST_ERR_SHAPE;
    return CAST_OK;
}

struct Call {
    const uint16_t* hidden;
    const uint16_t* weight;
    const int32_t* labels;
    uint16_t* grad_hidden;
    uint16_t* grad_weight;
    int64_t tokens, vocab, dim;
    uint8_t* ws;
    const Layout* l;
    cudaStream_t stream;
    int sms;
};

// The three products of one piece of tokens [t0, t0 + n).
template <int CG, int BN>
int exp_product(const Call& c, int64_t t0, int64_t n)
{
    const Layout& l = *c.l;
    CUtensorMap ma, mb;
    Shape s;
    ExpEpi epi;
    int rc;
    const bool grads = c.grad_hidden || c.grad_weight;
    if ((rc = make_shape<CG, BN, false, false, ExpEpi>(&s, true, n, c.vocab, c.dim, 1, 1, 16 / CG)) != CAST_OK) return rc;
    if ((rc = operand_map<false>(&ma, c.hidden + t0 * c.dim, n, c.dim, 1, c.dim, 0, 128)) != CAST_OK) return rc;
    if ((rc = operand_map<false>(&mb, c.weight, c.vocab, c.dim, 1, c.dim, 0, BN / CG)) != CAST_OK) return rc;
    epi.refs = reinterpret_cast<const float*>(c.ws + l.refs) + t0;
    epi.labels = c.labels + t0;
    epi.sums = reinterpret_cast<float*>(c.ws + l.sums);
    epi.tops = reinterpret_cast<float*>(c.ws + l.tops);
    epi.write_e = grads;
    epi.map_e = ma;
    if (grads && (rc = make_map(&epi.map_e, c.ws + l.e, 2, c.vocab, n, 1, l.e_ld, 0, 64, 32, true)) != CAST_OK) return rc;
    return launch<CG, BN, false, false>(ma, mb, s, epi, c.stream);
}

template <int CG, int BN>
int hidden_product(const Call& c, int64_t t0, int64_t n)
{
    const Layout& l = *c.l;
    CUtensorMap ma, mb;
    Shape s;
    HiddenGradEpi epi;
    int rc;
    const int splits = hidden_splits(n, c.vocab, c.dim, c.sms);
    if ((rc = make_shape<CG, BN, false, true, HiddenGradEpi>(&s, true, n, c.dim, c.vocab, 1, splits, 16 / CG)) != CAST_OK) return rc;
    if ((rc = operand_map<false>(&ma, c.ws + l.e, n, c.vocab, 1, l.e_ld, 0, 128)) != CAST_OK) return rc;
    if ((rc = operand_map<true>(&mb, c.weight, c.dim, c.vocab, 1, c.dim, 0, BN / CG)) != CAST_OK) return rc;
    epi.a = reinterpret_cast<const float*>(c.ws + l.a) + t0;
    epi.b = reinterpret_cast<const float*>(c.ws + l.b) + t0;
    epi.labels = c.labels + t0;
    epi.weight = c.weight;
    epi.vocab = (int)c.vocab;
    epi.partial = s.splits > 1;
    float* partial = reinterpret_cast<float*>(c.ws + l.partial);
    if (epi.partial) rc = make_map(&epi.map_out, partial, 4, c.dim, n, s.splits, c.dim, (uint64_t)n * c.dim, 32, 32, true);
    else rc = make_map(&epi.map_out, c.grad_hidden + t0 * c.dim, 2, c.dim, n, 1, c.dim, 0, 64, 32, true);
    if (rc != CAST_OK) return rc;
    if ((rc = launch<CG, BN, false, true>(ma, mb, s, epi, c.stream)) != CAST_OK) return rc;
    if (epi.partial) {
        const int64_t units = n * (c.dim / 8);
        return launch_chained(false, join_hidden_grad_kernel, dim3((unsigned)((units + kJoinThreads - 1) / kJoinThreads)), kJoinThreads, 0, c.stream, 1, partial, epi.a, epi.b,
                              epi.labels, c.weight, c.grad_hidden + t0 * c.dim, n, (int)c.dim, (int)c.vocab, s.splits);
    }
    return CAST_OK;
}

int weight_product(const Call& c, int64_t n, bool first, bool last)
{
    constexpr int CG = 2, BN = 256;
    const Layout& l = *c.l;
    CUtensorMap ma, mb;
    Shape s;
    WeightGradEpi epi;
    int rc;
    if ((rc = make_shape<CG, BN, true, true, WeightGradEpi>(&s, true, c.vocab, c.dim, n, 1, 1, 8)) != CAST_OK) return rc;
    if ((rc = operand_map<true>(&ma, c.ws + l.e, c.vocab, n, 1, l.e_ld, 0, 128)) != CAST_OK) return rc;
    if ((rc = operand_map<true>(&mb, c.ws + l.scaled, c.dim, n, 1, c.dim, 0, BN / CG)) != CAST_OK) return rc;
    epi.acc = reinterpret_cast<const float*>(c.ws + l.acc);
    epi.rows = reinterpret_cast<const float*>(c.ws + l.rows);
    epi.row_of = reinterpret_cast<const int32_t*>(c.ws + l.row_of);
    epi.add = !first;
    epi.last = last;
    if ((rc = make_map(&epi.map_out, c.grad_weight, 2, c.dim, c.vocab, 1, c.dim, 0, 64, 32, true)) != CAST_OK) return rc;
    epi.map_acc = epi.map_out;
    if (l.pieces > 1 && (rc = make_map(&epi.map_acc, c.ws + l.acc, 4, c.dim, c.vocab, 1, c.dim, 0, 32, 32, true)) != CAST_OK) return rc;
    return launch<CG, BN, true, true>(ma, mb, s, epi, c.stream);
}

}  // namespace
}  // namespace cast

using namespace cast;

extern "C" int cast_linear_ce_workspace(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece_tokens, int want_hidden_grad,
                                        int want_weight_grad, uint64_t* bytes)
{
    if (!bytes) return CAST_ERR_NULL;
    int rc, sms;
    if ((rc = check_ce_shape(tokens, vocab, dim, piece_tokens)) != CAST_OK) return rc;
    if ((rc = product::sm_count(&sms)) != CAST_OK) return rc;
    Layout l;
    if ((rc = layout_of(tokens, vocab, dim, piece_tokens, want_hidden_grad != 0, want_weight_grad != 0, sms, &l)) != CAST_OK) return rc;
    *bytes = l.total;
    return CAST_OK;
}

extern "C" int cast_linear_ce(const cast_bf16* hidden, const cast_bf16* weight, const int32_t* labels, float* loss, cast_bf16* grad_hidden,
                              cast_bf16* grad_weight, int64_t tokens, int64_t vocab, int64_t dim, float grad_scale, int64_t piece_tokens,
                              void* workspace, uint64_t workspace_bytes, cast_stream_t stream)
{
    if (!hidden || !weight || !labels || !loss || !workspace) return CAST_ERR_NULL;
    int rc;
    if ((rc = check_ce_shape(tokens, vocab, dim, piece_tokens)) != CAST_OK) return rc;
    if (!std::isfinite(grad_scale)) return CAST_ERR_HYPER;
    if (((uintptr_t)hidden | (uintptr_t)weight | (uintptr_t)grad_hidden | (uintptr_t)grad_weight | (uintptr_t)workspace) & 15u) return CAST_ERR_ALIGN;
    if (((uintptr_t)labels | (uintptr_t)loss) & 3u) return CAST_ERR_ALIGN;
    const uint64_t th = 2ull * (uint64_t)tokens * (uint64_t)dim, vw = 2ull * (uint64_t)vocab * (uint64_t)dim, t4 = 4ull * (uint64_t)tokens;
    int sms;
    if ((rc = product::sm_count(&sms)) != CAST_OK) return rc;
    Layout l;
    if ((rc = layout_of(tokens, vocab, dim, piece_tokens, grad_hidden != nullptr, grad_weight != nullptr, sms, &l)) != CAST_OK) return rc;
    if (workspace_bytes < l.total) return CAST_ERR_PLAN;
    const void* in[3] = {hidden, weight, labels};
    const uint64_t in_bytes[3] = {th, vw, t4};
    const void* out[4] = {loss, grad_hidden, grad_weight, workspace};
    const uint64_t out_bytes[4] = {t4, th, vw, l.total};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 3; ++j)
            if (ranges_overlap(out[i], out_bytes[i], in[j], in_bytes[j])) return CAST_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(out[i], out_bytes[i], out[j], out_bytes[j])) return CAST_ERR_ALIAS;
    }
    const void* ptrs[7] = {hidden, weight, labels, loss, grad_hidden, grad_weight, workspace};
    if ((rc = check_device_memory(ptrs, 7)) != CAST_OK) return rc;

    uint8_t* ws = static_cast<uint8_t*>(workspace);
    cudaStream_t st = (cudaStream_t)stream;
    const Call c = {hidden, weight, labels, grad_hidden, grad_weight, tokens, vocab, dim, ws, &l, st, sms};
    float* refs = reinterpret_cast<float*>(ws + l.refs);
    float* a = reinterpret_cast<float*>(ws + l.a);
    float* b = reinterpret_cast<float*>(ws + l.b);
    const unsigned own = (unsigned)((tokens + kRankThreads / 32 - 1) / (kRankThreads / 32));
    const SortStart start = sort_start(ws + l.scatter, tokens, dim);
    const unsigned fill0 = own + (grad_weight ? (unsigned)rank_blocks(tokens) : 0u);
    const unsigned fills = grad_weight ? (unsigned)((vocab + 4 * kRankThreads - 1) / (4 * kRankThreads)) : 0u;
    int32_t* row_of = reinterpret_cast<int32_t*>(ws + l.row_of);
    if ((rc = launch_chained(true, target_logit_kernel, dim3(fill0 + fills), kRankThreads, 0, st, 1, hidden, weight, labels, refs, tokens, (int)vocab,
                             (int)dim, own, fill0, start, reinterpret_cast<int4*>(row_of))) != CAST_OK)
        return rc;
    SortedTokens sorted;      // the merges now, while the ids are in L2, not after the products have swept it
    if (grad_weight && (rc = sort_tokens(true, labels, tokens, vocab, dim, ws + l.scatter, &sorted, st)) != CAST_OK) return rc;
    for (int64_t i = 0; i < l.pieces; ++i) {
        const int64_t t0 = i * l.piece, n = tokens - t0 < l.piece ? tokens - t0 : l.piece;
        rc = paired(n) ? exp_product<2, 256>(c, t0, n) : exp_product<1, 128>(c, t0, n);
        if (rc != CAST_OK) return rc;
        FinishArgs f;
        f.hidden = hidden + t0 * dim;
        f.labels = labels + t0;
        f.refs = refs + t0;
        f.sums = reinterpret_cast<const float*>(ws + l.sums);
        f.tops = reinterpret_cast<const float*>(ws + l.tops);
        f.loss = loss + t0;
        const bool grads = grad_hidden || grad_weight;
        f.a = grads ? a + t0 : nullptr;
        f.b = grads ? b + t0 : nullptr;
        f.e = grads ? reinterpret_cast<uint16_t*>(ws + l.e) : nullptr;
        f.scaled = grad_weight ? reinterpret_cast<uint16_t*>(ws + l.scaled) : nullptr;
        f.tokens = n;
        f.e_ld = l.e_ld;
        f.vocab = (int)vocab;
        f.dim = (int)dim;
        f.tile_cols = (int)tile_cols(n);
        f.n_tiles = (int)sum_rows(vocab, n);
        f.grad_scale = grad_scale;
        if ((rc = launch_chained(false, finish_kernel, dim3((unsigned)((n + kFinishTokens - 1) / kFinishTokens)), 256, 0, st, 1, f)) != CAST_OK) return rc;
        if (grad_hidden) {
            rc = paired(n) ? hidden_product<2, 256>(c, t0, n) : hidden_product<1, 128>(c, t0, n);
            if (rc != CAST_OK) return rc;
        }
        // b holds s S / (1 + S): the label's term of dW is -b H
        if (grad_weight && i + 1 == l.pieces &&
            (rc = gather_rows(sorted, hidden, b, reinterpret_cast<float*>(ws + l.rows), row_of, vocab, dim, st)) != CAST_OK)
            return rc;
        if (grad_weight && (rc = weight_product(c, n, i == 0, i + 1 == l.pieces)) != CAST_OK) return rc;
    }
    return CAST_OK;
}
