// Element-wise pieces of the operators over tokens.
#ifndef RTOSS_TOK_MATH_CUH
#define RTOSS_TOK_MATH_CUH

#include <type_traits>

#include "conv_common.cuh"

namespace rtoss_tok {

// Pairs of values: one instruction for both.
__device__ __forceinline__ unsigned long long& bits2(float2& v) { return reinterpret_cast<unsigned long long&>(v); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(bits2(d)) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(bits2(d)) : "l"(bits2(a)), "l"(bits2(b)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(bits2(d)) : "l"(bits2(a)), "l"(bits2(b)));
    return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Two neighbouring 16-bit values as they lie in a word.  (bf16: by shift and mask.  The conversion of a single value goes through the
// special-function pipe, which then bounds an elementwise kernel.)
template <typename T> __device__ __forceinline__ float2 widen2(unsigned w);
template <> __device__ __forceinline__ float2 widen2<__nv_bfloat16>(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
template <> __device__ __forceinline__ float2 widen2<__half>(unsigned w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// Pair j of eight values.
template <typename T, typename Eight>
__device__ __forceinline__ float2 pair_of(const Eight& v, int j) {
    if constexpr (sizeof(T) == 4) return make_float2(v.e[2 * j], v.e[2 * j + 1]);
    else return widen2<T>(reinterpret_cast<const unsigned*>(&v)[j]);
}

// f(std::integral_constant<int, ACT>): the activation is decided once for a run of elements
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    if (act == RTOSS_ACT_SILU) f(std::integral_constant<int, RTOSS_ACT_SILU>());
    else if (act == RTOSS_ACT_RELU) f(std::integral_constant<int, RTOSS_ACT_RELU>());
    else f(std::integral_constant<int, RTOSS_ACT_NONE>());
}

// 1 / (1 + e^-v) in the two special-function instructions it takes (2 ulp and 1 ulp).  Flushing subnormals costs nothing here: a
// subnormal exponential vanishes beside the 1, and below -88, where the exponential overflows, the quotient is the 0 it should
// be.  (__expf and __fdividef keep subnormals, at twice the time of an epilogue.)
__device__ __forceinline__ float sigmoid(float v) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}

// NaN goes through every activation.
template <int ACT>
__device__ __forceinline__ float act_of(float v) {
    if (ACT == RTOSS_ACT_RELU) return v < 0.f ? 0.f : v;
    if (ACT == RTOSS_ACT_SILU) return v * sigmoid(v);
    return v;
}
// Value and derivative (ReLU: 0 at 0).
template <int ACT>
__device__ __forceinline__ float act_slope(float v, float* slope) {
    if (ACT == RTOSS_ACT_RELU) {
        *slope = v > 0.f ? 1.f : 0.f;
        return v < 0.f ? 0.f : v;
    }
    if (ACT == RTOSS_ACT_SILU) {
        const float s = sigmoid(v);
        *slope = s + v * s * (1.f - s);
        return v * s;
    }
    *slope = 1.f;
    return v;
}
// One output of the 8-bit product: the exact integer sum, its two scales, bias, activation and residual, in fp32.
template <int ACT>
__device__ __forceinline__ float i8_value(int sum, float row_scale, float col_scale, float bias, float residual, int res_after) {
    const float v = fmaf((float)sum * row_scale, col_scale, bias);
    return res_after ? act_of<ACT>(v) + residual : act_of<ACT>(v + residual);
}

}  // namespace rtoss_tok

#endif
