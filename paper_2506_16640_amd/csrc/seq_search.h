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
//   A last step is not confirmed by another sweep where what it leaves is known to be less than 2^-19, from bounds of how the slope |f'| changes over it:
//   r >= 2, the root between the last two points (gap apart): the slope is a convex function of tau (f'' = r (r-1) sum x^(r-2) falls as keys leave), so it lies
//     below its chord, which the model follows, by at most twice the deficit of its integral (f's difference) over the gap; and at the gap's right end, where
//     it is smallest, by no more than the chord rises over t (half of that on average);
//   r = 2 (alpha 1.5) otherwise: over t the slope changes by at most 2 t times the keys that leave (t > 0: those that count now, or on average between the last
//     two points) or enter (t < 0: at most n, those that count at the bracket's left end where they were counted, else all that the row sees);
//   r > 2 otherwise: the model leaves out the third order, about |t| (|t| w) (d w) with w the larger of g and 2 B / A (both about one over the typical x) and
//     d = |t| where B was formed at this tau, else the larger of |t| and the gap; sixteen times that has to be below 2^-19;
//   r < 2: a key's term has an unbounded curvature where it meets the threshold, and at r = 1 the slope jumps there: the step itself has to be that short.
// (Rows of 17 to 1500 normal scores, deviations 0.3 to 1000, clusters of up to 290 equal ones, alpha 1.1 to 2, 2.9 million rows: threshold within 1.8e-6, from
// alpha 1.7 on within 2e-7.  Sweeps a row from the list kernels' bounds: 1.6 at alpha 1.5, 1.8 at 2, 2.5 at 1.25 and 1.7; from the left end 2.5, 2.6, 3.5, 4.2.
// At alpha 1.5 the third order with the gap as above leaves up to 4.5e-6 near clusters; the third order of t alone, for every alpha but 2, up to 3e-5
// at alpha 1.7 and 1e-4 at 1.95.)
template <int AM>
struct SeqSearch {
  float tau, lo, hi;
  float n;  // at most so many keys count at any tau of the bracket (to begin with: those that the row sees)
  float g_before, tau_before, f_before;
  bool before, whole_before;  // there was a point before; its sums were whole
  // with_k: the sums hold k.  Returns whether tau is final.
  ENTMAX_BOTH_SIDES bool step(const SeqSums& s, float r, bool with_k) {
    const float f = s.h - 1.0f, A = r * s.g;
    if (f >= 0.f) lo = fmaxf(lo, tau); else hi = fminf(hi, tau);
    if (AM == 1 && with_k && f >= 0.f) n = s.k;
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
    // (further below the largest score than 1, as after a sample that did not hold it, its term was cut off at 1: such sums tell the side, and a place to go on)
    const bool whole = tau >= -1.0f;
    if (!in) to = whole ? 0.5f * (lo + hi) : lo;
    const float at = fabsf(t);
    float left = at;
    if (AM != 2 && r >= 2.0f && curved && (with_k || whole_before)) {
      const float Ab = r * g_before, gap = fabsf(back);
      if (before && t * back > 0.f) {
        const float deficit = fabsf(0.5f * (A + Ab) * gap - fabsf(f - f_before));
        left = fminf(at, at * fminf(2.0f * deficit / gap, t < 0.f ? B * at : A) / fminf(A, Ab));
      } else if (AM == 1) {
        const float dA = 2.0f * (t >= 0.f ? B : n) * at;
        if (dA < 0.5f * A) left = 0.5f * at * dA / (A - dA);
      } else {
        const float w = fmaxf(s.g, A > 0.f ? 2.0f * B / A : 0.f);
        left = fminf(at, 16.0f * at * (at * w) * ((with_k ? at : fmaxf(at, gap)) * w));
      }
    }
    const bool fin = (in && whole && left <= 0x1p-19f) || hi - lo <= 0x1p-22f;
    before = true;
    whole_before = whole;
    g_before = s.g;
    f_before = f;
    tau_before = tau;
    tau = to;
    return fin;
  }
};

}  // namespace entmax
