// The 4-bit storage format shared by the weight matrices and the key/value cache (include/coreinfer.h
// section (7)): codes in units of two bytes, one fp16 pair (s, o) per group, x^ = s c + o.
#pragma once

#include "common.cuh"

namespace coreinfer {

constexpr float kHalfMax = 65504.f;

static inline bool group_known(int g) { return g == 32 || g == 64 || g == 128; }
static inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#ifdef __CUDACC__

// Typed views of the three storage types.
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Byte of the unit that holds values v .. v + 3 (v a multiple of 4) of a row piece of 32 H values.
__device__ __forceinline__ int unit_offset(int v, int H) { return 2 * (((v & 31) >> 2) * H + (v >> 5)); }

// Minimum, maximum and "holds a NaN" over the LANES consecutive lanes (a power of two) of a group.
template <int LANES>
__device__ __forceinline__ void group_range(float& lo, float& hi, bool& nan)
{
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        nan |= __shfl_xor_sync(0xffffffffu, (int)nan, d) != 0;
    }
}

// The pair of a group from its range.  Every step is one correctly rounded operation, so the format
// is a function of the values alone, whoever computes it.
struct QuantPair {
    __half s, o;
};
__device__ __forceinline__ QuantPair quant_pair(float lo, float hi, bool nan)
{
    QuantPair p;
    p.o = __float2half_rn(fminf(fmaxf(lo, -kHalfMax), kHalfMax));
    p.s = __float2half_rn(fminf(__fdiv_rn(__fsub_rn(hi, lo), 15.f), kHalfMax));
    if (nan) p.s = p.o = __ushort_as_half((unsigned short)0x7fff);
    return p;
}
// (x - o) / s with s <= 0 or NaN: code 0.
__device__ __forceinline__ unsigned quant_code(float x, float s, float o)
{
    if (!(s > 0.f)) return 0u;
    return (unsigned)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x, o), s)), 0.f), 15.f);
}

#endif  // __CUDACC__

}  // namespace coreinfer
