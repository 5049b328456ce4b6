// Activations and their slopes in fp32, for the epilogue of the forward product and the pass in front of the backward one.
#pragma once
#include <type_traits>

#include "osdp_internal.h"

namespace osdp {
namespace {

// 2^x and 1 / x as the hardware has them: off by one unit in the last place.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

constexpr float kLog2e = 1.44269504088896341f;
// gelu_tanh: 0.5 z (1 + tanh u) = z sigma(2 u) with 2 u = z (kTanhA + kTanhB z^2): no cancellation for negative z.
constexpr float kTanhA = 1.59576912160573f, kTanhB = 1.59576912160573f * 0.044715f;
constexpr float kInvSqrt2Pi = 0.398942280401433f;

// 1 / (1 + exp(-x)); exp(-x) beyond the range gives 0.
__device__ __forceinline__ float sigmoid(float x) { return fast_rcp(1.0f + fast_exp2(-kLog2e * x)); }

// Phi(-a) exp(a^2 / 2) for a >= 0, Phi the normal distribution: t times a polynomial in t = 1 / (1 + 0.28 a), fitted to
// erfcx(a / sqrt 2) / 2 by least squares, reweighted until the relative error is level: at most 3.7e-6 for all a, 4.1e-6 with the
// roundings in fp32.  Times the exponential, the roundings of whose argument count a^2 / 2 fold, the tails are off by 4.4e-6 of
// themselves for a below 6, 7e-6 below 9 and 1.1e-5 up to 13, where 1 - erf would keep nothing.
__device__ __forceinline__ float normal_tail_scaled(float a) {
  const float t = fast_rcp(__builtin_fmaf(0.28f, a, 1.0f));
  float q = -0.050230203738183314f;
  q = __builtin_fmaf(q, t, 0.10544056629310301f);
  q = __builtin_fmaf(q, t, 0.024952666947975228f);
  q = __builtin_fmaf(q, t, 0.09445458859018137f);
  q = __builtin_fmaf(q, t, 0.10193606019244618f);
  q = __builtin_fmaf(q, t, 0.11174063934621645f);
  q = __builtin_fmaf(q, t, 0.1117038440438022f);
  return q * t;
}

// act(z).  NaN stays NaN; z of -infinity gives NaN, as z times 0 does, but for none and relu.
template <int kAct>
__device__ __forceinline__ float activate(float z) {
  if constexpr (kAct == OSDP_ACT_RELU) return __builtin_elementwise_maximum(z, 0.0f);  // (NaN stays: v_maximum3)
  if constexpr (kAct == OSDP_ACT_GELU) {
    const float e = fast_exp2((-0.5f * kLog2e) * z * z), tail = e * normal_tail_scaled(__builtin_fabsf(z));
    return z * (z < 0.0f ? tail : 1.0f - tail);
  }
  if constexpr (kAct == OSDP_ACT_GELU_TANH) return z * sigmoid(z * __builtin_fmaf(kTanhB, z * z, kTanhA));
  if constexpr (kAct == OSDP_ACT_SILU) return z * sigmoid(z);
  return z;
}

// act'(z); relu: 1 for z > 0 and for NaN, else 0.
template <int kAct>
__device__ __forceinline__ float activation_slope(float z) {
  if constexpr (kAct == OSDP_ACT_RELU) return z <= 0.0f ? 0.0f : 1.0f;
  if constexpr (kAct == OSDP_ACT_GELU) {
    const float e = fast_exp2((-0.5f * kLog2e) * z * z), tail = e * normal_tail_scaled(__builtin_fabsf(z));
    return __builtin_fmaf(z, e * kInvSqrt2Pi, z < 0.0f ? tail : 1.0f - tail);
  }
  if constexpr (kAct == OSDP_ACT_GELU_TANH) {
    // (beyond 20 the slope is 0 or 1 to the last bit, and the cube would leave the range; 0 z keeps NaN)
    const float c = __builtin_amdgcn_fmed3f(z, -20.0f, 20.0f), c2 = c * c;
    const float s = sigmoid(c * __builtin_fmaf(kTanhB, c2, kTanhA));
    const float slope = __builtin_fmaf(c * s * (1.0f - s), __builtin_fmaf(3.0f * kTanhB, c2, kTanhA), s);
    return __builtin_fmaf(0.0f, z, slope);
  }
  if constexpr (kAct == OSDP_ACT_SILU) {
    const float s = sigmoid(z);
    return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
  }
  return 1.0f;
}

// f(an integral constant) with the launch's activation, which all lanes share, as a compile-time number.
template <class F>
__device__ __forceinline__ void with_activation(int act, F &&f) {
  switch (act) {
    case OSDP_ACT_RELU: f(std::integral_constant<int, OSDP_ACT_RELU>{}); break;
    case OSDP_ACT_GELU: f(std::integral_constant<int, OSDP_ACT_GELU>{}); break;
    case OSDP_ACT_GELU_TANH: f(std::integral_constant<int, OSDP_ACT_GELU_TANH>{}); break;
    case OSDP_ACT_SILU: f(std::integral_constant<int, OSDP_ACT_SILU>{}); break;
    default: f(std::integral_constant<int, OSDP_ACT_NONE>{}); break;
  }
}

__device__ __forceinline__ float bf16_low(uint32_t two) { return __builtin_bit_cast(float, two << 16); }
__device__ __forceinline__ float bf16_high(uint32_t two) { return __builtin_bit_cast(float, two & 0xffff0000u); }

}  // namespace
}  // namespace osdp
