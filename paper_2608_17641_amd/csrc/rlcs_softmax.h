// Device building blocks of the kernels over rows of logits and of attention: softmax statistics in
// base 2, their joins over lanes and waves, and keys that order floats as unsigned integers.
#pragma once

#include "rlcs_device.h"

namespace rlcs {

// One workgroup a row, as a grid of two axes: a launch counts the lanes of each in 32 bits, which 2^23 rows
// of 512 lanes would pass.
constexpr int kGridBits = 20;
inline dim3 row_grid(int64_t rows) {
    const int64_t x = int64_t(1) << kGridBits;
    return rows <= x ? dim3(unsigned(rows)) : dim3(unsigned(x), unsigned((rows + x - 1) >> kGridBits));
}
__device__ __forceinline__ int64_t grid_row() { return (int64_t(blockIdx.y) << kGridBits) + blockIdx.x; }

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff(), kNegInf = -kInf;

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

// Logarithms of weights are kept from -inf, whose product with a weight of 0 is NaN: 2^-150 is 0.
constexpr float kLog2Zero = -150.f;

// Weights of a row whose largest element is `top`: 2^((x - top) c), with c = log2(e) / temperature. The
// difference is exact where it counts. Of -inf alone (above() gives them a top of 0) all weights are 0;
// next to +inf or NaN they are NaN.
struct Above {
    float top, c;
    __device__ __forceinline__ float log2_weight(float x) const { return (x - top) * c; }
};
__device__ __forceinline__ Above above(float top, float c) { return Above{top == kNegInf ? 0.f : top, c}; }

// The same with one operation: 2^(x c - m), m = top c. The fused multiply-add rounds once, and the
// rounding of m, up to 64 below 2^31, is a factor common to every element, which cancels in a softmax.
// From 2^31 on whatever differs from top at all is at least 128 below it in base 2: a power of two
// in c's place, with which m is exact, tells the elements equal to top (2^0) from the others (less
// than 2^-64).
struct Scale {
    float c, m;
    __device__ __forceinline__ float log2_weight(float x) const { return fmaf(x, c, -m); }
};
__device__ __forceinline__ Scale scale_of(float top, float c) {
    const float m = top * c;
    if (fabsf(m) < 2147483648.f) return Scale{c, m};
    if (top == kNegInf) return Scale{kInf, 0.f};
    const int e = 126 - ilogbf(top), of_c = ilogbf(c);
    const float p = ldexpf(1.f, of_c < e ? of_c : e);
    return Scale{p, top * p};
}
// Logarithm of the factor from weights of one top to those of a larger one: by the rounded m, as those
// are what the weights are relative to. Tops of different c are far apart.
__device__ __forceinline__ float scale_step(const Scale& from, const Scale& to) {
    return from.c == to.c ? fmaxf(from.m - to.m, kLog2Zero) : kLog2Zero;
}

// Over each group of L lanes, every lane with the result; the tree is fixed, so the sums are too.
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
template <int L>
__device__ __forceinline__ float max_lanes(float v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// Over the whole wave: within rows of 16 lanes by row shifts, across them by two broadcasts (DPP moves of
// the vector unit, a few clocks each, where a shuffle goes through LDS); lane 63 has the result,
// which a lane read hands to all. f(a, b) with `id` its neutral element.
template <class T, class F>
__device__ __forceinline__ T fold_wave(T v, T id, F&& f) {
    constexpr int kWords = sizeof(T) / 4;
    struct Words {
        int w[kWords];
    };
    auto step = [&](auto ctrl, auto rows) {
        const Words x = __builtin_bit_cast(Words, v), n = __builtin_bit_cast(Words, id);
        Words o;
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            o.w[i] = __builtin_amdgcn_update_dpp(n.w[i], x.w[i], decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        v = f(v, __builtin_bit_cast(T, o));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});  // row_shr:1
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // row_bcast:15
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // row_bcast:31
    Words x = __builtin_bit_cast(Words, v);
#pragma unroll
    for (int i = 0; i < kWords; ++i) x.w[i] = __builtin_amdgcn_readlane(x.w[i], 63);
    return __builtin_bit_cast(T, x);
}
__device__ __forceinline__ float sum_wave(float v) {
    return fold_wave(v, 0.f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float max_wave(float v) {
    return fold_wave(v, kNegInf, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ uint64_t max_wave(uint64_t v) {
    return fold_wave(v, uint64_t(0), [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}

// 16 bytes of a row, at any element address.
template <typename DT>
struct RowVec {
    static constexpr int K = 16 / sizeof(DT);
    typedef typename std::conditional<sizeof(DT) == 4, u32x4_any, u32x4_any2>::type Any;
    u32x4 w;
    // Vector i of a row of V elements: whole, or the row's end with -inf after it.
    __device__ __forceinline__ void load(const DT* x, int64_t i, int64_t V) {
        if ((i + 1) * K <= V) {
            w = *reinterpret_cast<const Any*>(x + i * K);
        } else {
            const uint32_t inf = sizeof(DT) == 4 ? 0xff800000u : 0xff80ff80u;
            w = u32x4{inf, inf, inf, inf};
            for (int k = 0; i * K + k < V; ++k) {
                if constexpr (sizeof(DT) == 4) {
                    const uint32_t e = reinterpret_cast<const uint32_t*>(x)[i * K + k];
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[q] = k == q ? e : w[q];
                } else {
                    const uint32_t e = reinterpret_cast<const uint16_t*>(x)[i * K + k];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (k >> 1 == q) w[q] = (k & 1) ? (w[q] & 0xffffu) | (e << 16) : (w[q] & 0xffff0000u) | e;
                }
            }
        }
    }
    __device__ __forceinline__ float at(int k) const {
        if constexpr (sizeof(DT) == 4) return __uint_as_float(w[k]);
        else return __uint_as_float((k & 1) ? (w[k >> 1] & 0xffff0000u) : (w[k >> 1] << 16));
    }
};

// Writes vector i of a row of V elements.
template <typename DT>
__device__ __forceinline__ void store_row_vec(DT* x, int64_t i, int64_t V, const float (&v)[16 / sizeof(DT)]) {
    constexpr int K = 16 / sizeof(DT);
    u32x4 w;
    if constexpr (sizeof(DT) == 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __float_as_uint(v[k]);
    } else {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < 4; ++k)
            w[k] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(v[2 * k]), static_cast<__bf16>(v[2 * k + 1])});
    }
    if ((i + 1) * K <= V) {
        __builtin_nontemporal_store(w, reinterpret_cast<typename RowVec<DT>::Any*>(x + i * K));
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (i * K + k < V) x[i * K + k] = narrow(v[k], DT{});
    }
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
