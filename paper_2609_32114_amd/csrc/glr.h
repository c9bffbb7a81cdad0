// glr.h -- the gate of the recurrence: the decay a and its complement 1 - a from a
// log-gate or a raw projection.
#pragma once

#include "device.h"

namespace hagdn {

struct Gate {
  float a, forget;  // decay e^g, and 1 - a
};

// RAW: g holds a raw value r, the log-gate being -softplus(r): a = 1 / (1 + e^r) and
// 1 - a = 1 / (1 + e^-r), both from e^-|r| so that nothing overflows and neither
// loses digits.  Else a = e^g, and 1 - a = -g (1 + g/2 (1 + g/3 (...))) near zero,
// where 1 - e^g would cancel: the series' first seven terms, whose remainder is
// under 2^-25 of the sum for |g| <= 0.35.
// The exponential is the hardware's 2^x of one product: its relative error is
// |g| 2^-24 from the product and an ulp of its own, which a, falling as e^g, hides.
template <bool RAW> __device__ __forceinline__ Gate glr_gate(float g) {
  constexpr float kLog2e = 1.44269504f;
  Gate k;
  if constexpr (RAW) {
    const float t = __builtin_amdgcn_exp2f(-__builtin_fabsf(g) * kLog2e);
    const float r = __builtin_amdgcn_rcpf(1.f + t), tr = t * r;
    k.a = g > 0.f ? tr : r;
    k.forget = g > 0.f ? r : tr;
  } else {
    k.a = __builtin_amdgcn_exp2f(g * kLog2e);
    float p = 1.f + g * (1.f / 7.f);
    p = 1.f + g * (1.f / 6.f) * p;
    p = 1.f + g * (1.f / 5.f) * p;
    p = 1.f + g * (1.f / 4.f) * p;
    p = 1.f + g * (1.f / 3.f) * p;
    p = 1.f + g * (1.f / 2.f) * p;
    k.forget = __builtin_fabsf(g) <= 0.35f ? -g * p : 1.f - k.a;
  }
  return k;
}

}  // namespace hagdn
