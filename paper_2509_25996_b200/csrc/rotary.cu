// Rotary positions with one or several axes: pair i of every head of token t turns by frequencies[i] * positions[axes[i]][t],
//   (a, b) -> (a cos - b sin, a sin + b cos),
// and by minus that for the gradient.  Pairs are (i, i + pairs) or, adjacent, (2i, 2i + 1).
//
// Bounded by HBM: every entry is read and written once.  A CTA takes a few tokens and some of their heads: its threads ask for their
// entries first, work out the cosines and sines of the CTA's tokens while those travel, and share them through shared memory, so that an angle is
// worked out once for all heads.
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
constexpr int kItems = 4;                 // units that a thread has in flight
constexpr int kBatch = kTurnThreads * kItems;
constexpr int kAngles = 1024;             // cosines and sines of a CTA (8 KB)
constexpr int kMostUnits = 16384;         // of a CTA

// i / d for i < 2^16, d < 2^16
struct Divisor {
    uint32_t d, magic;
};
Divisor divisor(uint32_t d) { return {d, d > 1 ? (uint32_t)(0x100000000ull / d + 1) : 0u}; }
__device__ __forceinline__ uint32_t divide(uint32_t i, Divisor v) { return v.d > 1 ? __umulhi(i, v.magic) : i; }

struct HeadSet {
    const uint16_t* in;
    uint16_t* out;
    int64_t in_token, in_head, out_token, out_head;     // strides in entries
    int32_t first;                                       // heads of the sets before it
};

struct RotaryArgs {
    HeadSet set[kMostSets];
    const double* frequencies;
    const int32_t* axes;              // or NULL: all on axis 0
    const int32_t* positions;         // [n_axes][tokens]
    int32_t sets, heads;              // heads of all sets together
    int32_t tokens, n_axes, pairs;
    int32_t turned;                   // units of a head that turn; each holds W pairs (halves) or W columns (adjacent)
    Divisor units;                    // and with those that are copied
    Divisor token_units;              // of a token in a CTA (of the last CTA of a token's heads: fewer)
    Divisor pair_count;
    int32_t tile_tokens, tile_heads;  // of a CTA
    int32_t head_tiles;
    float sign;
};

// W: columns per access.  Halves: a unit is W columns of the first half and the W of the second that go with them.
template <int W, bool ADJACENT>
__global__ void __launch_bounds__(kTurnThreads)
rotary_kernel(const __grid_constant__ RotaryArgs a)
{
    // one column per access cannot hold an adjacent pair: two accesses then, too
    constexpr bool TWO = !ADJACENT || W == 1;
    constexpr int P = W == 1 ? 1 : ADJACENT ? W / 2 : W;        // pairs of a unit
    using A = Access<W>;
    using Raw = typename A::Raw;
    // [token][pair of a unit / 2][unit][2]: neighbouring units, which neighbouring threads hold, lie side by side
    __shared__ __align__(16) float2 angle[kAngles];
    const int64_t token0 = (int64_t)(blockIdx.x / a.head_tiles) * a.tile_tokens;
    const int head0 = (int)(blockIdx.x % a.head_tiles) * a.tile_heads;
    const int tokens = (int)min((int64_t)a.tile_tokens, a.tokens - token0), heads = min(a.tile_heads, a.heads - head0);
    const uint32_t total = (uint32_t)tokens * (uint32_t)heads * a.units.d;
    Raw x[kItems], y[TWO ? kItems : 1];
    uint16_t* dst[kItems];
    int place[kItems];                    // of the unit's first angles, -1: a copy, -2: none
    auto fetch = [&](uint32_t first) {
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const uint32_t i = first + threadIdx.x + k * kTurnThreads;
            place[k] = -2;
            if (i >= total) continue;
            // several tokens only with all of their heads: token_units is theirs then
            const uint32_t t = a.tile_tokens > 1 ? divide(i, a.token_units) : 0u, rest = i - t * a.token_units.d, hd = divide(rest, a.units);
            const int u = (int)(rest - hd * a.units.d), head = head0 + (int)hd;
            int s = 0;
            while (s + 1 < a.sets && head >= a.set[s + 1].first) ++s;
            const HeadSet& hs = a.set[s];
            const int64_t token = token0 + t, own = head - hs.first;
            const bool turns = u < a.turned;
            const int col = turns ? (ADJACENT ? u * 2 * P : u * W) : 2 * a.pairs + (u - a.turned) * W;      // the unit's first column
            const uint16_t* src = hs.in + token * hs.in_token + own * hs.in_head + col;
            dst[k] = hs.out + token * hs.out_token + own * hs.out_head + col;
            place[k] = turns ? (int)t * a.pairs + u * (P > 1 ? 2 : 1) : -1;
            x[k] = *reinterpret_cast<const Raw*>(src);
            if constexpr (TWO)
                if (turns) y[k] = *reinterpret_cast<const Raw*>(src + (ADJACENT ? 1 : a.pairs));
        }
    };
    fetch(0);
    for (uint32_t i = threadIdx.x; i < (uint32_t)(tokens * a.pairs); i += kTurnThreads) {
        const uint32_t t = divide(i, a.pair_count), p = i - t * a.pairs;
        const uint32_t axis = a.axes ? (uint32_t)__ldg(a.axes + p) : 0u;
        float2 cs = make_float2(1.0f, 0.0f);              // a pair of no axis does not turn
        if (axis < (uint32_t)a.n_axes) {
            const double turns = (double)__ldg(a.positions + (int64_t)axis * a.tokens + token0 + t) * (__ldg(a.frequencies + p) * 0.15915494309189533577);
            sincospif(2.0f * (float)(turns - rint(turns)), &cs.y, &cs.x);
            cs.y *= a.sign;
        }
        angle[t * a.pairs + (P > 1 ? (p % P / 2 * a.turned + p / P) * 2 + p % 2 : p)] = cs;
    }
    __syncthreads();
    for (uint32_t first = 0;;) {
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            if (place[k] == -2) continue;
            if (place[k] == -1) {
                *reinterpret_cast<Raw*>(dst[k]) = x[k];
                continue;
            }
            float u[W], v[W];
            A::unpack(x[k], u);
            if constexpr (TWO) A::unpack(y[k], v);
#pragma unroll
            for (int j = 0; j < P; j += 2) {
                float4 cs;
                if constexpr (P > 1) {
                    cs = *reinterpret_cast<const float4*>(angle + place[k] + j * a.turned);
                } else {
                    const float2 one = angle[place[k]];
                    cs = make_float4(one.x, one.y, 0.0f, 0.0f);
                }
#pragma unroll
                for (int e = 0; e < (P > 1 ? 2 : 1); ++e) {
                    const float c = e ? cs.z : cs.x, s = e ? cs.w : cs.y;
                    float& p = TWO ? u[j + e] : u[(2 * (j + e)) % W];
                    float& q = TWO ? v[j + e] : u[(2 * (j + e) + 1) % W];
                    const float p0 = p, q0 = q;
                    p = p0 * c - q0 * s;
                    q = p0 * s + q0 * c;
                }
            }
            *reinterpret_cast<Raw*>(dst[k]) = A::pack(u);
            if constexpr (TWO) *reinterpret_cast<Raw*>(dst[k] + (ADJACENT ? 1 : a.pairs)) = A::pack(v);
        }
        first += kBatch;
        if (first >= total) break;
        fetch(first);
    }
}

template <int W, bool ADJACENT>
int launch_rotary(RotaryArgs a, int64_t head_dim, int sms, cudaStream_t stream)
{
    a.turned = W == 1 ? a.pairs : ADJACENT ? 2 * a.pairs / W : a.pairs / W;
    const int units = a.turned + (int)((head_dim - 2 * a.pairs) / W);
    // Several tokens per CTA, so that their angles keep its threads busy, but not so many that SMs stay idle; a token of more units
    // than a batch is shared by CTAs where there are few tokens, and where its units exceed a CTA's most.
    const int64_t token_units = (int64_t)a.heads * units, wanted = (int64_t)sms * 8;
    a.tile_heads = a.heads;
    a.tile_tokens = 1;
    if (token_units > kMostUnits || (token_units > kBatch && a.tokens < wanted)) {
        const int64_t pieces = (token_units + kBatch - 1) / kBatch;
        a.tile_heads = (int)((a.heads + pieces - 1) / pieces);
    } else {
        int64_t most = kAngles / a.pairs;
        if (most > kMostUnits / token_units) most = kMostUnits / token_units;
        if (most > 4096 / token_units + 1) most = 4096 / token_units + 1;
        if (most > a.tokens / wanted) most = a.tokens / wanted;
        if (most > 1) a.tile_tokens = (int)most;
    }
    a.units = divisor((uint32_t)units);
    a.token_units = divisor((uint32_t)(a.tile_heads * units));
    a.pair_count = divisor((uint32_t)a.pairs);
    a.head_tiles = (a.heads + a.tile_heads - 1) / a.tile_heads;
    const int64_t grid = (int64_t)((a.tokens + a.tile_tokens - 1) / a.tile_tokens) * a.head_tiles;
    if (grid > 0x7FFFFFFF) return CAST_ERR_SHAPE;
    rotary_kernel<W, ADJACENT><<<(unsigned)grid, kTurnThreads, 0, stream>>>(a);
    CAST_CUDA_TRY(cudaGetLastError());
    count_launch();
    return CAST_OK;
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
    bool vec = head_dim % 8 == 0 && pairs % (adjacent ? 4 : 8) == 0;
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
        // strides up to 2^40 entries: products with the counts fit 64 bits
        const int64_t strides[4] = {s.in_token_stride, s.in_head_stride, s.out_token_stride, s.out_head_stride};
        for (int j = 0; j < 4; ++j)
            if (strides[j] < 0 || strides[j] > ((int64_t)1 << 40) / (j % 2 ? s.heads : tokens)) return CAST_ERR_SHAPE;
        if (!apart(tokens, s.heads, head_dim, s.out_token_stride, s.out_head_stride)) return CAST_ERR_SHAPE;
        if (((uintptr_t)s.in & 1u) || ((uintptr_t)s.out & 1u)) return CAST_ERR_ALIGN;
        vec = vec && !((uintptr_t)s.in & 15u) && !((uintptr_t)s.out & 15u);
        for (int j = 0; j < 4; ++j) vec = vec && strides[j] % 8 == 0;
        in_bytes[i] = span_bytes(tokens, s.heads, head_dim, s.in_token_stride, s.in_head_stride);
        out_bytes[i] = span_bytes(tokens, s.heads, head_dim, s.out_token_stride, s.out_head_stride);
        a.set[i] = {s.in, s.out, s.in_token_stride, s.in_head_stride, s.out_token_stride, s.out_head_stride, (int32_t)heads};
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
    a.sign = inverse ? -1.0f : 1.0f;
    const cudaStream_t st = (cudaStream_t)stream;
    int device = 0, sms = 0;
    CAST_CUDA_TRY(cudaGetDevice(&device));
    CAST_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    if (vec) return adjacent ? launch_rotary<8, true>(a, head_dim, sms, st) : launch_rotary<8, false>(a, head_dim, sms, st);
    return adjacent ? launch_rotary<1, true>(a, head_dim, sms, st) : launch_rotary<1, false>(a, head_dim, sms, st);
}
