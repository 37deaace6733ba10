// Element-wise pieces of the operators over tokens.
#ifndef RTOSS_TOK_MATH_CUH
#define RTOSS_TOK_MATH_CUH

#include <type_traits>

#include "conv_common.cuh"

namespace rtoss_tok {

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
