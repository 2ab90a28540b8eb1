// Device building blocks of the kernels over rows of logits and of attention: softmax statistics in
// base 2, their joins over lanes and waves, and keys that order floats as unsigned integers.
#pragma once

#include "rlcs_device.h"

namespace rlcs {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();

// v_exp_f32 and v_log_f32: base 2, 1 ulp.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

__device__ __forceinline__ bf16_t narrow(float x, bf16_t) {  // to nearest, ties to even
    uint32_t u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return bf16_t{uint16_t((u >> 16) | 0x40u)};
    u += 0x7fffu + ((u >> 16) & 1u);
    return bf16_t{uint16_t(u >> 16)};
}
__device__ __forceinline__ float narrow(float x, float) { return x; }

// Weights of a row whose largest element is `top`: 2^(x c - m), with c = log2(e) / temperature and
// m = top c. The fused multiply-add of x c - m rounds once, and the rounding of m is common to
// every element, so it cancels in a softmax. Where top c overflows, whatever differs from top at all
// is at least 2^100 below it in base 2: a power of two in c's place, with which top c is
// exact, tells the elements equal to top (2^0) from the others (0).
struct Scale {
    float c, m;
    __device__ __forceinline__ float log2_weight(float x) const { return fmaf(x, c, -m); }
};
__device__ __forceinline__ Scale scale_of(float top, float c) {
    const float m = top * c;
    if (fabsf(m) < __builtin_inff() || top == kNegInf) return Scale{c, m};
    const float p = ldexpf(1.f, 126 - ilogbf(top));
    return Scale{p, top * p};
}

__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float max_lanes(float v) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// Floats as unsigned keys in the same order (-0 as +0; NaN as -inf).
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint((x == x ? x : kNegInf) + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

}  // namespace rlcs
