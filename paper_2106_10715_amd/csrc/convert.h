// Device helpers shared by the kernels around the expert layer: 16-byte pieces, bf16 and e4m3 conversions, sums and
// maxima over neighbouring lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moe {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kE4M3Max = 448.f;
constexpr float kMinScale = 0x1p-126f;      // a row of zeros has a scale too, and 1 / scale is finite

// Two values to bf16, to the nearest, ties to even.
__device__ inline uint32_t to_bf16x2(float lo, float hi) {
    const bf16x2 r = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ inline float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ inline float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// Four values to e4m3, to the nearest, ties to even; |v| may not pass 448 by more than rounding, NaN stays NaN.
__device__ inline uint32_t to_e4m3x4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}
__device__ inline void from_e4m3x4(uint32_t u, float (&v)[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), true);
    v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1];
}

// The scale of values whose largest magnitude is `top`.
__device__ inline float e4m3_scale(float top) { return fmaxf(top / kE4M3Max, kMinScale); }

// v / scale for the values of one scale, rounded to the nearest.  A product with the rounded 1 / scale alone is off by a bit in a quarter of all
// cases, which at a border between two e4m3 values is a whole step: here 1 / scale has what its rounding left out beside it, 46 bits in all
// (fewer for scales past 2^100, at least 30).  v / infinity is 0 for finite v.  16384 tokens of 8 x 128 written:
// 19.3 us, with the product alone 18.9, corrected by the remainder 20.4, divided 24.8.
struct OverScale {
    float inv, rest;
    __device__ explicit OverScale(float scale) : inv(1.f / scale), rest(inv == 0.f ? 0.f : fmaf(-inv, scale, 1.f) * inv) {}
    __device__ float operator()(float v) const { return fmaf(v, inv, v * rest); }
};

// Loads and stores that leave the caches to others, where STREAM says so.
template <bool STREAM, typename T>
__device__ inline T load_from(const T* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool STREAM, typename T>
__device__ inline void store_to(T* p, T v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Sum and maximum over each run of N neighbouring lanes (N a power of two up to 64), in all of its lanes.
template <int N>
__device__ inline float lanes_sum(float v) {
#pragma unroll
    for (int o = 1; o < N; o *= 2) v += __shfl_xor(v, o);
    return v;
}
template <int N>
__device__ inline float lanes_max(float v) {
#pragma unroll
    for (int o = 1; o < N; o *= 2) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

}  // namespace moe
