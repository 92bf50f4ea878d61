// Activations of the gated block: value and derivative.
#ifndef FW_GATED_ACT_CUH_
#define FW_GATED_ACT_CUH_

#include "fw_rows.cuh"

namespace fw {

// 1 / (1 + exp(-x)): 0 and 1 at the ends, NaN for NaN
__device__ __forceinline__ float logistic(float x) {
  return rows::rcp(1.f + rows::ex2(-1.4426950408889634f * x));
}

template <int ACT>
struct Act {
  // f = act(a), df = act'(a)
  static __device__ __forceinline__ void both(float a, float& f, float& df) {
    if (ACT == FW_ACT_SILU) {
      const float p = logistic(a);
      f = a * p;
      df = fmaf(f, 1.f - p, p);
    } else if (ACT == FW_ACT_GELU) {
      const float cdf = 0.5f * erfcf(-0.70710678118654752f * a);
      f = a * cdf;
      df = fmaf(a * 0.3989422804014327f, rows::ex2(-0.72134752044448170f * a * a), cdf);
    } else if (ACT == FW_ACT_GELU_TANH) {
      // (1 + tanh(x)) / 2 = logistic(2 x)
      // (the square is kept finite: p is 0 or 1 long before, and 0 times infinity is no derivative; a NaN goes on through f)
      const float k = 1.5957691216057308f, a2 = fminf(a * a, 1e30f);
      const float p = logistic(k * a * fmaf(0.044715f, a2, 1.f));
      f = a * p;
      df = fmaf(f * (1.f - p), k * fmaf(0.134145f, a2, 1.f), p);
    } else {
      f = a > 0.f || a != a ? a : 0.f;
      df = a > 0.f ? 1.f : a != a ? a : 0.f;
    }
  }
  static __device__ __forceinline__ float value(float a) {
    float f, df;
    both(a, f, df);
    return f;
  }
};

// body(Act<...>{}) for the activation `act`: the choice is made outside of the loops
template <class F>
__device__ __forceinline__ void with_act(int act, F&& body) {
  if (act == FW_ACT_SILU) body(Act<FW_ACT_SILU>{});
  else if (act == FW_ACT_GELU) body(Act<FW_ACT_GELU>{});
  else if (act == FW_ACT_GELU_TANH) body(Act<FW_ACT_GELU_TANH>{});
  else body(Act<FW_ACT_RELU>{});
}

}  // namespace fw
#endif
