// The tiled serving kernel's search for a row's threshold from sums over all its keys, sweep by sweep.  Plain C++: the kernel's own code is also run on
// the CPU by the tests.
#pragma once
#include <math.h>

#if defined(__HIPCC__)
#define ENTMAX_BOTH_SIDES __host__ __device__ __forceinline__
#else
#define ENTMAX_BOTH_SIDES inline
#endif

namespace entmax {

// Sums over a row's keys at tau, x = [y - tau]_+:  g = sum x^(r-1), h = sum x^r, and in the first sweep of alpha 1.5 and 1.25 k = sum x^(r-2).
struct SeqSums {
  float g, h, k;
};

// y and tau are taken relative to the row's largest score, so that tau lies in [-1, 0) and its last place is 2^-24 whatever the size of the scores.
// f = h - 1, f' = -r g; half the curvature, B, comes from k where it was formed, else from the change of g since the sweep before.  A step t goes to the
// root of the quadratic model, inside the bracket [lo, hi].
//   No sweep is spent on confirming the last step.  The model leaves out the third order: after a step t about t^3 w^2 is left, w the larger of g and
// 2 B / A (both about one over the typical x), without a curvature t^2 w r / 2; a step that leaves less than 2^-20 by 64 times (16 times) that ends the
// search.  At alpha 2, where f is piecewise linear and its curvature jumps from key to key, the last step is confirmed.
template <int AM>
struct SeqSearch {
  float tau, lo, hi;
  float g_before, tau_before;
  bool before;
  // with_k: the sums hold k.  Returns whether tau is final.
  ENTMAX_BOTH_SIDES bool step(const SeqSums& s, float r, bool with_k) {
    const float f = s.h - 1.0f, A = r * s.g;
    if (f >= 0.f) lo = fmaxf(lo, tau); else hi = fminf(hi, tau);
    const float back = tau_before - tau;
    float B = 0.f;
    bool curved = false;
    if (AM != 2 && with_k) {
      B = 0.5f * r * (r - 1.0f) * s.k;
      curved = true;
    } else if (AM != 2 && before && back != 0.f) {
      B = fmaxf(0.5f * r * (s.g - g_before) / back, 0.f);
      curved = true;
    }
    const float t = 2.0f * f / (A + sqrtf(fmaxf(fmaf(A, A, -4.0f * B * f), 0.f)));
    float to = tau + t;
    const bool in = A > 0.f && to >= lo && to <= hi;
    if (!in) to = 0.5f * (lo + hi);
    const float at = fabsf(t), w = fmaxf(s.g, A > 0.f ? 2.0f * B / A : 0.f);
    const float left = AM == 2 ? at : (curved ? 64.0f * at * (at * w) * (at * w) : 8.0f * at * (at * w) * r);
    const bool fin = (in && left <= 0x1p-20f) || hi - lo <= 0x1p-22f;
    before = true;
    g_before = s.g;
    tau_before = tau;
    tau = to;
    return fin;
  }
};

}  // namespace entmax
