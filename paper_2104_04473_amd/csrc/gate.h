// Activations of the gated feed-forward block and their derivatives, shared by the element-wise kernels and the GEMMs' output stages:
// g = f(a) c, and with dg: da = dg f'(a) c, dc = dg f(a); a, c: the gate's and the up projection's sum with its bias.
#pragma once
#include "gelu.h"
#include <type_traits>

namespace ptdp {

// 1 / (1 + exp(-a)) with the hardware's exponential and reciprocal (1 ulp each; exp overflowing to infinity gives exactly 0)
__device__ __forceinline__ float sigmoid_f(float a) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -1.4426950408889634f)); }
template <int GATE> __device__ __forceinline__ float gate_f(float a) {
  if (GATE == PTDP_GATE_SILU) return a * sigmoid_f(a);
  if (GATE == PTDP_GATE_GELU_ERF) return gelu_f<PTDP_GELU_ERF>(a);
  if (GATE == PTDP_GATE_GELU_TANH) return gelu_f<PTDP_GELU_TANH>(a);
  if (GATE == PTDP_GATE_SIGMOID) return sigmoid_f(a);
  return a > 0.f || a != a ? a : 0.f;   // (an undefined element stays one)
}
// f(a), and f'(a) to *d
template <int GATE> __device__ __forceinline__ float gate_grad_f(float a, float* d) {
  if (GATE == PTDP_GATE_GELU_ERF) {
    float pdf;
    const float cdf = normal_cdf_pdf(a, &pdf);
    *d = cdf + a * pdf;
    return a * cdf;
  }
  if (GATE == PTDP_GATE_GELU_TANH) {
    const float c = 0.7978845608028654f, th = fast_tanh(c * (a + 0.044715f * a * a * a));
    *d = 0.5f * (1.f + th) + 0.5f * a * (1.f - th * th) * c * (1.f + 3.f * 0.044715f * a * a);
    return 0.5f * a * (1.f + th);
  }
  if (GATE == PTDP_GATE_RELU) {
    *d = a > 0.f ? 1.f : 0.f;
    return a > 0.f || a != a ? a : 0.f;
  }
  const float s = sigmoid_f(a);
  if (GATE == PTDP_GATE_SIGMOID) {
    *d = s * (1.f - s);
    return s;
  }
  *d = s * (1.f + a * (1.f - s));
  return a * s;
}
// calls f with std::integral_constant<int, gate>
template <class F> __host__ __device__ __forceinline__ void with_gate(int gate, F&& f) {
  switch (gate) {
    case PTDP_GATE_SILU: f(std::integral_constant<int, PTDP_GATE_SILU>{}); break;
    case PTDP_GATE_GELU_ERF: f(std::integral_constant<int, PTDP_GATE_GELU_ERF>{}); break;
    case PTDP_GATE_GELU_TANH: f(std::integral_constant<int, PTDP_GATE_GELU_TANH>{}); break;
    case PTDP_GATE_SIGMOID: f(std::integral_constant<int, PTDP_GATE_SIGMOID>{}); break;
    default: f(std::integral_constant<int, PTDP_GATE_RELU>{});
  }
}

}  // namespace ptdp
