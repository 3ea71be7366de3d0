// Accesses of 8 bf16 columns (16 bytes) or of one, and their conversions, shared by the norm, the rotary positions and the clipping.
#pragma once

#include <stdint.h>

namespace cast {

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// W columns of one access: `Raw` as they lie in memory.
template <int W> struct Access;
template <> struct Access<8> {
    using Raw = uint4;
    static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
    static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[8])
    {
        v[0] = bf16_low(r.x); v[1] = bf16_high(r.x); v[2] = bf16_low(r.y); v[3] = bf16_high(r.y);
        v[4] = bf16_low(r.z); v[5] = bf16_high(r.z); v[6] = bf16_low(r.w); v[7] = bf16_high(r.w);
    }
    static __device__ __forceinline__ Raw pack(const float (&v)[8])
    {
        return make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
    // weights: W entries of a bf16 or fp32 vector
    static __device__ __forceinline__ void weights(const uint16_t* p, float (&v)[8]) { unpack(__ldg(reinterpret_cast<const uint4*>(p)), v); }
    static __device__ __forceinline__ void weights(const float* p, float (&v)[8])
    {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
template <> struct Access<1> {
    using Raw = uint16_t;
    static __device__ __forceinline__ Raw zero() { return 0; }
    static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[1]) { v[0] = bf16_low(r); }
    static __device__ __forceinline__ Raw pack(const float (&v)[1]) { return (Raw)(bf16_pair(v[0], 0.0f) & 0xFFFFu); }
    static __device__ __forceinline__ void weights(const uint16_t* p, float (&v)[1]) { v[0] = bf16_low(__ldg(p)); }
    static __device__ __forceinline__ void weights(const float* p, float (&v)[1]) { v[0] = __ldg(p); }
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// The columns of a 16-byte access as pairs.
struct Pairs {
    static __device__ __forceinline__ void unpack(const uint4& r, float2 (&v)[4])
    {
        v[0] = make_float2(bf16_low(r.x), bf16_high(r.x)); v[1] = make_float2(bf16_low(r.y), bf16_high(r.y));
        v[2] = make_float2(bf16_low(r.z), bf16_high(r.z)); v[3] = make_float2(bf16_low(r.w), bf16_high(r.w));
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&v)[4])
    {
        return make_uint4(bf16_pair(v[0].x, v[0].y), bf16_pair(v[1].x, v[1].y), bf16_pair(v[2].x, v[2].y), bf16_pair(v[3].x, v[3].y));
    }
    static __device__ __forceinline__ void weights(const uint16_t* p, float2 (&v)[4]) { unpack(__ldg(reinterpret_cast<const uint4*>(p)), v); }
    static __device__ __forceinline__ void weights(const float* p, float2 (&v)[4])
    {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        v[0] = make_float2(a.x, a.y); v[1] = make_float2(a.z, a.w); v[2] = make_float2(b.x, b.y); v[3] = make_float2(b.z, b.w);
    }
};

}  // namespace cast
