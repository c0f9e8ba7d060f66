// Activations of the gated layer and their derivatives, in fp32.
#pragma once

#include "gl_device.h"

namespace gl {

enum { kActNone = 0, kActGelu = 1, kActSilu = 2 };  // gl_act

// Phi(-a) e^(a^2 / 2) for a >= 0 falls like 1 / a for large a: with t = 1 / (1 + p a) it is
// t q(t), q a smooth function on (0, 1].  q is a polynomial fitted in float64 to the least
// largest error relative to Phi(-a), weighted by what the output's type shows of it, so
// that the tail's small results have their bits too:
//   bf16  five terms, within 5.7e-7 e^(1.5 a), never more than 2.8e-3 (2^-8 is its rounding)
//   fp32  eight terms, within 3.8e-8 (1 + a)
// The three terms more would cost a bf16 gated layer up to 2.7 % (12544 x 640 x 2560 94.4 us for
// 97.0 without pre, 16384 x 2048 x 4096 443 for 446, 6272 x 192 x 768 and single rows nothing);
// down to -4, where the GELU is -1.3e-4, five are within a sixteenth of its type's rounding.
template <int DT>
__device__ __forceinline__ float gauss_tail(float a) {
  const float t = __builtin_amdgcn_rcpf(fmaf(DT ? 0.34400001f : 0.3f, a, 1.f));
  float q;
  if (DT) {
    q = fmaf(t, -0.100211024f, 0.2995327891f);
    q = fmaf(t, q, -0.005176517668f);
    q = fmaf(t, q, 0.1722774513f);
    q = fmaf(t, q, 0.1335771899f);
  } else {
    q = fmaf(t, 0.03661797821f, -0.1609455123f);
    q = fmaf(t, q, 0.212445229f);
    q = fmaf(t, q, -0.0589276667f);
    q = fmaf(t, q, 0.1311242333f);
    q = fmaf(t, q, 0.09920725217f);
    q = fmaf(t, q, 0.1208549423f);
    q = fmaf(t, q, 0.1196235572f);
  }
  return t * q;
}

// e^(-x^2 / 2)
__device__ __forceinline__ float gauss_exp(float x) {
  const float y = x * 0.84932180028801907f;  // sqrt(log2(e) / 2)
  return __builtin_amdgcn_exp2f(-y * y);
}

// GELU x Phi(x) = max(x, 0) - |x| Phi(-|x|), with its limits at the infinities.
template <int DT>
__device__ __forceinline__ float gelu_tail(float x) {
  const float a = fabsf(x);
  const float tq = gauss_tail<DT>(a), e = gauss_exp(x);
  return fmaf(-fminf(a, 3.4e38f), tq * e, fmaxf(x, 0.f));
}

// 1 / (1 + e^-x); the division by a reciprocal of about one unit in the last place.  Below
// 2^-126, x < -87.3, it is 0: the hardware's reciprocal gives no subnormals.
__device__ __forceinline__ float sigmoid_f32(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
}

// The gate's activation of N values (uniform `act`, asked once: behind a branch for each value
// their chains of instructions would run one after the other); x sigmoid(x) is 0 at -infinity.
template <int DT, int N>
__device__ __forceinline__ void gate_acts(int act, float (&x)[N]) {
  if (act == kActGelu) {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = gelu_tail<DT>(x[j]);
  } else if (act == kActSilu) {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = fmaxf(x[j], -3.4e38f) * sigmoid_f32(x[j]);
  }
}

// The activation, in place, and its derivative:
//   GELU  Phi(x) + x e^(-x^2 / 2) / sqrt(2 pi)
//   SiLU  s + x s (1 - s), s = sigmoid(x); 1 - s is sigmoid(-x), which keeps its bits
template <int N>
__device__ __forceinline__ void gate_act_grads(int act, float (&x)[N], float (&da)[N]) {
  if (act == kActGelu) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float a = fminf(fabsf(x[j]), 3.4e38f), e = gauss_exp(x[j]), tail = gauss_tail<0>(a) * e;
      const float c = a * e * 0.3989422804014327f;
      da[j] = x[j] < 0.f ? tail - c : 1.f - tail + c;
      x[j] = fmaf(-a, tail, fmaxf(x[j], 0.f));
    }
  } else if (act == kActSilu) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float s = sigmoid_f32(x[j]), c = fmaxf(fminf(x[j], 3.4e38f), -3.4e38f) * s;
      da[j] = fmaf(c, sigmoid_f32(-x[j]), s);
      x[j] = fmaxf(x[j], -3.4e38f) * s;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) da[j] = 1.f;
  }
}

}  // namespace gl
