// Rotary positions with one or several axes: pair i of every head of token t turns by frequencies[i] * positions[axes[i]][t],
//   (a, b) -> (a cos - b sin, a sin + b cos),
// and by minus that for the gradient.  Pairs are (i, i + pairs) or, adjacent, (2i, 2i + 1).
//
// Bounded by HBM: every entry is read and written once.  A CTA takes a few tokens and some of their heads: its threads ask for their
// entries first, work out the cosines and sines of the CTA's tokens while those travel, and share them through shared memory, so that an angle is
// worked out once for all heads.  16384 tokens of 32 + 32 heads of 128 columns 81.5 us (537 MB, 6.6 TB/s), 87 under the power limit; of 32 + 8 heads
// 52.1; 8190 tokens of 48 heads with adjacent pairs 36.5 us (201 MB, 5.5 TB/s): one access per thread and unit, so that addresses and
// angles weigh twice as much (71 % of the issue slots busy).
//
// Angles are formed in fp64 as turns and reduced to half a turn before they become fp32: a position of 2^20 times a frequency of one
// radian would lose its turn in fp32.  Cosine and sine, the products and their sum are fp32; results are rounded once.
#include "bf16_access.cuh"
#include "chained.cuh"
#include "embed.cuh"

namespace cast {
namespace {

constexpr int kMostSets = 4;              // arrays of heads turned by one call (queries, keys, ...)
constexpr int kMostPairs = 512;
constexpr int kTurnThreads = 256;
constexpr int kAngles = 1024;             // cosines and sines of a CTA (8 KB)

// i / d for i < 2^16, d < 2^16
struct Divisor {
    uint32_t d, magic;
};
Divisor divisor(uint32_t d) { return {d, d > 1 ? (uint32_t)(0x100000000ull / d + 1) : 0u}; }
__device__ __forceinline__ uint32_t divide(uint32_t i, Divisor v) { return v.d > 1 ? __umulhi(i, v.magic) : i; }

struct HeadSet {
    const uint16_t* in;
    uint16_t* out;
    int32_t in_token, in_head, out_token, out_head;     // strides in entries
    int32_t first;                                       // heads of the sets before it
};

struct RotaryArgs {
    HeadSet set[kMostSets];
    const double* frequencies;
    const int32_t* axes;              // or NULL: all on axis 0
    const int32_t* positions;         // [n_axes][tokens]
    int32_t sets, heads;              // heads of all sets together
    int32_t tokens, n_axes, pairs, head_dim;
    int32_t turned;                   // units of a head that turn
    Divisor units;                    // and with those that are copied
    Divisor token_units;              // of a token in a CTA
    Divisor pair_count;
    int32_t tile_tokens, tile_heads;  // of a CTA
    int32_t head_tiles;
    float sign;
};

// W bf16 columns of one access, as words of two (W == 1: one in the low half)
template <int W> struct Words { uint32_t w[W > 1 ? W / 2 : 1]; };
template <int W>
__device__ __forceinline__ Words<W> load_words(const uint16_t* p)
{
    Words<W> r;
    if constexpr (W == 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else if constexpr (W == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        r.w[0] = v.x; r.w[1] = v.y;
    } else if constexpr (W == 2) {
        r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        r.w[0] = *p;
    }
    return r;
}
template <int W>
__device__ __forceinline__ void store_words(uint16_t* p, const Words<W>& r)
{
    if constexpr (W == 8) *reinterpret_cast<uint4*>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    else if constexpr (W == 4) *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
    else if constexpr (W == 2) *reinterpret_cast<uint32_t*>(p) = r.w[0];
    else *p = (uint16_t)r.w[0];
}

// A unit is what a thread turns of a head.  Halves: W columns of the first half and the W of the second that go with them.  Adjacent:
// W columns (of which the last turning unit may copy some), or with W == 1 two single ones.
template <int W, bool ADJACENT>
struct Unit {
    static constexpr bool kTwo = !ADJACENT || W == 1;                        // two accesses
    static constexpr int kPairs = ADJACENT ? (W == 1 ? 1 : W / 2) : W;
    static constexpr int kColumns = ADJACENT ? 2 * kPairs : W;               // from one unit's first column to the next one's
};

// ITEMS: units of a thread, all of them in flight.
template <int W, bool ADJACENT, int ITEMS>
__global__ void __launch_bounds__(kTurnThreads, ITEMS < 4 ? 6 : 5)
rotary_kernel(const __grid_constant__ RotaryArgs a)
{
    using U = Unit<W, ADJACENT>;
    constexpr int P = U::kPairs;
    // [token][pair of a unit / 2][unit][2]: neighbouring units, which neighbouring threads hold, lie side by side
    __shared__ __align__(16) float2 angle[kAngles];
    const int token0 = (int)(blockIdx.x / a.head_tiles) * a.tile_tokens;
    const int head0 = (int)(blockIdx.x % a.head_tiles) * a.tile_heads;
    const int tokens = min(a.tile_tokens, a.tokens - token0), heads = min(a.tile_heads, a.heads - head0);
    const uint32_t total = (uint32_t)tokens * (uint32_t)heads * a.units.d;
    Words<W> x[ITEMS], y[U::kTwo ? ITEMS : 1];
    uint16_t* dst[ITEMS];
    int place[ITEMS];                    // of the unit's first angles, -1: a copy, -3: a copy of one access, -2: none
    int left[ADJACENT && W == 8 ? ITEMS : 1];        // pairs that turn from the unit's first one on
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const uint32_t i = threadIdx.x + k * blockDim.x;
        place[k] = -2;
        if (i >= total) continue;
        // several tokens only with all of their heads: token_units is theirs then
        const uint32_t t = a.tile_tokens > 1 ? divide(i, a.token_units) : 0u, rest = i - t * a.token_units.d, hd = divide(rest, a.units);
        const int u = (int)(rest - hd * a.units.d), head = head0 + (int)hd;
        int s = 0;
        while (s + 1 < a.sets && head >= a.set[s + 1].first) ++s;
        const HeadSet& hs = a.set[s];
        const int64_t token = token0 + (int)t, own = head - hs.first;           // 32-bit factors of the strides
        const bool turns = u < a.turned;
        // the unit's first column; a copying unit takes as many accesses as a turning one
        const int col = turns ? u * U::kColumns : U::kTwo ? 2 * a.pairs + (u - a.turned) * 2 * W : u * W;
        const uint16_t* src = hs.in + token * hs.in_token + own * hs.in_head + col;
        dst[k] = hs.out + token * hs.out_token + own * hs.out_head + col;
        place[k] = turns ? (int)t * a.turned * P + u * (P > 1 ? 2 : 1) : U::kTwo && col + W < a.head_dim ? -1 : -3;
        x[k] = load_words<W>(src);
        if constexpr (U::kTwo)
            if (place[k] != -3) y[k] = load_words<W>(src + (!turns ? W : ADJACENT ? 1 : a.pairs));
        if constexpr (ADJACENT && W == 8) left[k] = a.pairs - u * P;
    }
    for (uint32_t i = threadIdx.x; i < (uint32_t)(tokens * a.pairs); i += blockDim.x) {
        const uint32_t t = divide(i, a.pair_count), p = i - t * a.pairs;
        const uint32_t axis = a.axes ? (uint32_t)__ldg(a.axes + p) : 0u;
        float2 cs = make_float2(1.0f, 0.0f);              // a pair of no axis does not turn
        if (axis < (uint32_t)a.n_axes) {
            const double turns = (double)__ldg(a.positions + (int64_t)axis * a.tokens + token0 + t) * (__ldg(a.frequencies + p) * 0.15915494309189533577);
            sincospif(2.0f * (float)(turns - rint(turns)), &cs.y, &cs.x);
            cs.y *= a.sign;
        }
        angle[t * a.turned * P + (P > 1 ? (p % P / 2 * a.turned + p / P) * 2 + p % 2 : p)] = cs;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        if (place[k] == -2) continue;
        if (place[k] >= 0) {
            if constexpr (W == 1) {
                const float2 cs = angle[place[k]];
                const float p = bf16_low(x[k].w[0]), q = bf16_low(y[k].w[0]);
                x[k].w[0] = bf16_pair(p * cs.x - q * cs.y, 0.0f);
                y[k].w[0] = bf16_pair(p * cs.y + q * cs.x, 0.0f);
            } else if constexpr (ADJACENT) {
                float2 cs[P];
                if constexpr (W == 8) {
#pragma unroll
                    for (int j = 0; j < P; j += 2) {
                        const float4 two = *reinterpret_cast<const float4*>(angle + place[k] + j * a.turned);
                        cs[j] = make_float2(two.x, two.y);
                        cs[j + 1] = make_float2(two.z, two.w);
                    }
                } else {
                    cs[0] = angle[place[k]];
                }
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float p = bf16_low(x[k].w[j]), q = bf16_high(x[k].w[j]);
                    const uint32_t turned = bf16_pair(p * cs[j].x - q * cs[j].y, p * cs[j].y + q * cs[j].x);
                    if (W < 8 || j < left[W == 8 ? k : 0]) x[k].w[j] = turned;
                }
            } else {
#pragma unroll
                for (int j = 0; j < W / 2; ++j) {
                    const float4 cs = *reinterpret_cast<const float4*>(angle + place[k] + 2 * j * a.turned);
                    const float2 c = make_float2(cs.x, cs.z), s = make_float2(cs.y, cs.w);
                    const float2 p = make_float2(bf16_low(x[k].w[j]), bf16_high(x[k].w[j])), q = make_float2(bf16_low(y[k].w[j]), bf16_high(y[k].w[j]));
                    const float2 u = fma2(p, c, mul2(q, make_float2(-s.x, -s.y))), v = fma2(p, s, mul2(q, c));
                    x[k].w[j] = bf16_pair(u.x, u.y);
                    y[k].w[j] = bf16_pair(v.x, v.y);
                }
            }
            if constexpr (U::kTwo) store_words<W>(dst[k] + (ADJACENT ? 1 : a.pairs), y[k]);
        } else if constexpr (U::kTwo) {
            if (place[k] == -1) store_words<W>(dst[k] + W, y[k]);
        }
        store_words<W>(dst[k], x[k]);
    }
}

template <int W, bool ADJACENT, int ITEMS>
int launch_items(RotaryArgs a, int units, int sms, cudaStream_t stream)
{
    using U = Unit<W, ADJACENT>;
    constexpr int kBatch = kTurnThreads * ITEMS;
    // No CTA goes round twice: those that did were slower the more rounds they made (16384 tokens of 64 heads of 128 columns, halves: 88 us,
    // with twice the tokens per CTA 98, with four times 104).  As many whole tokens as fit, or a part of one token's heads.
    const int64_t token_units = (int64_t)a.heads * units, slots = (int64_t)a.turned * U::kPairs;
    a.tile_heads = a.heads;
    a.tile_tokens = 1;
    if (token_units > kBatch) {
        // CTAs of about as many heads each; at least one fits, since a head has at most 1024 columns
        const int fit = kBatch / units, pieces = (a.heads + fit - 1) / fit;
        a.tile_heads = (a.heads + pieces - 1) / pieces;
    } else {
        int64_t most = kBatch / token_units;
        if (most > kAngles / slots) most = kAngles / slots;
        if (most > a.tokens / sms) most = a.tokens / sms;             // few tokens: a CTA each
        if (most > 1) a.tile_tokens = (int)most;
    }
    a.units = divisor((uint32_t)units);
    a.token_units = divisor((uint32_t)(a.tile_heads * units));
    a.pair_count = divisor((uint32_t)a.pairs);
    a.head_tiles = (a.heads + a.tile_heads - 1) / a.tile_heads;
    // threads for the units, or for the angles where those are more work (few heads)
    int64_t threads = ((int64_t)a.tile_tokens * a.tile_heads * units + ITEMS - 1) / ITEMS, of_angles = (int64_t)a.tile_tokens * a.pairs / 2;
    if (threads < of_angles) threads = of_angles;
    threads = threads > kTurnThreads ? kTurnThreads : (threads + 31) / 32 * 32;
    const int64_t grid = (int64_t)((a.tokens + a.tile_tokens - 1) / a.tile_tokens) * a.head_tiles;
    if (grid > 0x7FFFFFFF) return CAST_ERR_SHAPE;
    rotary_kernel<W, ADJACENT, ITEMS><<<(unsigned)grid, (unsigned)threads, 0, stream>>>(a);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    return CAST_OK;
}

template <int W, bool ADJACENT>
int launch_rotary(RotaryArgs a, int64_t head_dim, int sms, cudaStream_t stream)
{
    using U = Unit<W, ADJACENT>;
    a.turned = (a.pairs + U::kPairs - 1) / U::kPairs;
    constexpr int copied = U::kTwo ? 2 * W : W;          // columns of a unit
    const int units = a.turned + (int)((head_dim - (U::kTwo ? 2 * a.pairs : a.turned * W) + copied - 1) / copied);
    // Halves: two units, which are four 16-byte accesses, per thread and 6 CTAs per SM are enough (81.4 us for those 16384 tokens; four units
    // and 4 CTAs 82.6).  Adjacent units have one access: as many as keep a token in one CTA, which works out its angles once, and leave no
    // thread idle (8190 tokens of 48 heads of 128 columns: two 38.9 us, three 36.5, four 38.8; 16384 of 64: two 99.9, three 93.5, four 90.0).
    if constexpr (W == 8 && !ADJACENT) {
        return launch_items<W, ADJACENT, 2>(a, units, sms, stream);
    } else if constexpr (W == 8) {
        const int64_t token_units = (int64_t)a.heads * units;
        return token_units <= 2 * kTurnThreads   ? launch_items<W, ADJACENT, 2>(a, units, sms, stream)
               : token_units <= 3 * kTurnThreads ? launch_items<W, ADJACENT, 3>(a, units, sms, stream)
                                                 : launch_items<W, ADJACENT, 4>(a, units, sms, stream);
    } else {
        return launch_items<W, ADJACENT, 4>(a, units, sms, stream);
    }
}

// Bytes from the first to behind the last entry of `heads` heads of `tokens` tokens.
uint64_t span_bytes(int64_t tokens, int64_t heads, int64_t dim, int64_t token_stride, int64_t head_stride)
{
    return 2ull * (uint64_t)((tokens - 1) * token_stride + (heads - 1) * head_stride + dim);
}

// No two of the heads lie on one another (either order of the strides).
bool apart(int64_t tokens, int64_t heads, int64_t dim, int64_t token_stride, int64_t head_stride)
{
    if (heads > 1 && head_stride < dim) return false;
    if (tokens > 1 && token_stride < dim) return false;
    if (tokens == 1 || heads == 1) return true;
    return token_stride >= (heads - 1) * head_stride + dim || head_stride >= (tokens - 1) * token_stride + dim;
}

}  // namespace
}  // namespace cast

using namespace cast;

extern "C" int cast_rotary(const cast_heads_t* sets, int n_sets, const int32_t* positions, const double* frequencies, const int32_t* axes, int n_axes,
                           int pairs, int adjacent, int inverse, int64_t tokens, int64_t head_dim, cast_stream_t stream)
{
    if (!sets || !positions || !frequencies) return CAST_ERR_NULL;
    if (n_sets < 1 || n_sets > kMostSets || n_axes < 1 || n_axes > 64 || (n_axes > 1 && !axes)) return CAST_ERR_SHAPE;
    if (tokens < 1 || tokens > 0x3FFFFFFF || pairs < 1 || pairs > kMostPairs || head_dim < 2 * (int64_t)pairs || head_dim > 2 * kMostPairs) return CAST_ERR_SHAPE;
    if (((uintptr_t)positions & 3u) || ((uintptr_t)frequencies & 7u) || ((uintptr_t)axes & 3u)) return CAST_ERR_ALIGN;
    RotaryArgs a = {};
    // columns that every address, stride and count is a multiple of
    uint64_t common = 8u | (uint64_t)head_dim | (adjacent ? 0u : (uint64_t)pairs);
    const uint64_t table_bytes[3] = {4ull * (uint64_t)n_axes * (uint64_t)tokens, 8ull * (uint64_t)pairs, 4ull * (uint64_t)pairs};
    const void* const table[3] = {positions, frequencies, axes};
    cast_heads_t own[kMostSets];
    uint64_t in_bytes[kMostSets], out_bytes[kMostSets];
    const void* ptrs[3 + 2 * kMostSets] = {positions, frequencies, axes};
    int64_t heads = 0;
    for (int i = 0; i < n_sets; ++i) {
        cast_heads_t& s = own[i];
        s = sets[i];
        if (!s.in || !s.out) return CAST_ERR_NULL;
        // the stride of a single token or head counts for nothing
        if (tokens == 1) s.in_token_stride = s.out_token_stride = 0;
        if (s.heads == 1) s.in_head_stride = s.out_head_stride = 0;
        if (s.heads < 1 || s.heads > 65536) return CAST_ERR_SHAPE;
        const int64_t strides[4] = {s.in_token_stride, s.in_head_stride, s.out_token_stride, s.out_head_stride};
        for (int j = 0; j < 4; ++j)
            if (strides[j] < 0 || strides[j] > 0x7FFFFFFF) return CAST_ERR_SHAPE;
        if (!apart(tokens, s.heads, head_dim, s.out_token_stride, s.out_head_stride)) return CAST_ERR_SHAPE;
        if (((uintptr_t)s.in & 1u) || ((uintptr_t)s.out & 1u)) return CAST_ERR_ALIGN;
        common |= (uintptr_t)s.in / 2 | (uintptr_t)s.out / 2;
        for (int j = 0; j < 4; ++j) common |= (uint64_t)strides[j];
        in_bytes[i] = span_bytes(tokens, s.heads, head_dim, s.in_token_stride, s.in_head_stride);
        out_bytes[i] = span_bytes(tokens, s.heads, head_dim, s.out_token_stride, s.out_head_stride);
        a.set[i] = {s.in, s.out, (int32_t)s.in_token_stride, (int32_t)s.in_head_stride, (int32_t)s.out_token_stride, (int32_t)s.out_head_stride, (int32_t)heads};
        heads += s.heads;
        ptrs[3 + 2 * i] = s.in;
        ptrs[4 + 2 * i] = s.out;
    }
    // A result may take the place of its own input (same strides).  Sets may lie side by side in one array, e.g. the heads of a fused
    // projection: their spans meet although no entries do, as long as they share the token's stride.
    for (int i = 0; i < n_sets; ++i) {
        const cast_heads_t& o = own[i];
        for (int j = 0; j < 3; ++j)
            if (ranges_overlap(o.out, out_bytes[i], table[j], table_bytes[j])) return CAST_ERR_ALIAS;
        for (int j = 0; j < 2 * n_sets; ++j) {
            const cast_heads_t& s = own[j / 2];
            const bool out = j % 2 != 0;
            if (out && j / 2 == i) continue;
            const uint16_t* p = out ? s.out : s.in;
            const int64_t token = out ? s.out_token_stride : s.in_token_stride, head = out ? s.out_head_stride : s.in_head_stride;
            if (!out && j / 2 == i && p == o.out && token == o.out_token_stride && head == o.out_head_stride) continue;
            if (!ranges_overlap(o.out, out_bytes[i], p, out ? out_bytes[j / 2] : in_bytes[j / 2])) continue;
            // rows of the same stride, each within one stride: apart if their places within the stride are
            const int64_t stride = o.out_token_stride, row_o = (o.heads - 1) * o.out_head_stride + head_dim, row_s = (s.heads - 1) * head + head_dim;
            if (token != stride || stride < 1) return CAST_ERR_ALIAS;
            const int64_t distance = ((intptr_t)p - (intptr_t)o.out) % (2 * stride), d = distance < 0 ? distance + 2 * stride : distance;
            if (d % 2 != 0 || d < 2 * row_o || d + 2 * row_s > 2 * stride) return CAST_ERR_ALIAS;
        }
    }
    if (heads > 65536) return CAST_ERR_SHAPE;
    int rc;
    if ((rc = check_device_memory(ptrs, 3 + 2 * n_sets)) != CAST_OK) return rc;
    a.frequencies = frequencies;
    a.axes = axes;
    a.positions = positions;
    a.sets = n_sets;
    a.heads = (int32_t)heads;
    a.tokens = (int32_t)tokens;
    a.n_axes = n_axes;
    a.pairs = pairs;
    a.head_dim = (int32_t)head_dim;
    a.sign = inverse ? -1.0f : 1.0f;
    const cudaStream_t st = (cudaStream_t)stream;
    int device = 0, sms = 0;
    CAST_CUDA_TRY(cudaGetDevice(&device));
    CAST_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    const int w = (int)(common & (~common + 1));          // the lowest bit: 1, 2, 4 or 8
    if (adjacent)
        return w == 8   ? launch_rotary<8, true>(a, head_dim, sms, st)
               : w >= 2 ? launch_rotary<2, true>(a, head_dim, sms, st)
                        : launch_rotary<1, true>(a, head_dim, sms, st);
    return w == 8   ? launch_rotary<8, false>(a, head_dim, sms, st)
           : w == 4 ? launch_rotary<4, false>(a, head_dim, sms, st)
           : w == 2 ? launch_rotary<2, false>(a, head_dim, sms, st)
                    : launch_rotary<1, false>(a, head_dim, sms, st);
}
