// The tiled serving kernel's threshold search (its own code) on rows of normal scores, many of them with clusters of equal ones, from the starts that the
// kernel has.  The sums are formed in 64 bits and rounded once, so that what is seen is the search.
//   The threshold: the search leaves at most 2^-19; f = h - 1 with h to half a step of 1 to 2 over a slope of at least 1 (the terms are at most 1 and their
//   powers r add up to 1, so their powers r - 1 add up to 1 at least), and tau's own last place: 2^-22 for both.
//   The sweeps: no row comes near the limit where the kernel gives up (48), and alpha 2 takes about as many as alpha 1.5.
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <random>
#include <vector>

#include "seq_search.h"

using namespace entmax;
using std::vector;

static std::mt19937_64 rng(7);
static std::normal_distribution<float> normal;

static SeqSums sums_at(const vector<float>& z, float tau, double r) {
  double g = 0, h = 0, k = 0;
  for (float y : z) {
    const double x = std::min(1.0, (double)y - (double)tau);
    if (x <= 0) continue;
    const double p = r == 1.0 ? 1.0 : (r == 2.0 ? x : pow(x, r - 1.0));
    g += p;
    h += p * x;
    k += r < 2.0 ? 0.0 : (r == 2.0 ? 1.0 : p / x);
  }
  return SeqSums{(float)g, (float)h, (float)k};
}

static double exact_tau(const vector<float>& z, double r) {
  double lo = -1.0, hi = 0.0;  // relative to the largest score
  for (int i = 0; i < 50; ++i) {
    const double mid = 0.5 * (lo + hi);
    double h = 0;
    for (float y : z)
      if (y > mid) h += r == 1.0 ? y - mid : (r == 2.0 ? (y - mid) * (y - mid) : pow(y - mid, r));
    (h >= 1.0 ? lo : hi) = mid;
  }
  return 0.5 * (lo + hi);
}

struct Seen {
  double sweeps = 0;
  int rows = 0, most = 0;
  double worst = 0;
};

// start 0: from a lower bound of the list kernels' kind (the threshold of the largest of every eight scores); 1: from the left end; 2: from an estimate near
// the threshold, on either side, and the largest score of a quarter of the keys
template <int AM>
static void row(float alpha, int n, int cluster, float deviation, int start, Seen& seen) {
  const float r = 1.0f / (alpha - 1.0f);
  vector<float> y(n);
  for (float& v : y) v = (alpha - 1.0f) * deviation * normal(rng);
  for (int i = 0; i < n; ++i) y[i] = y[i - i % cluster];
  std::shuffle(y.begin(), y.end(), rng);
  const float top = *std::max_element(y.begin(), y.end());
  vector<float> z(n);
  for (int i = 0; i < n; ++i) z[i] = y[i] - top;
  const double want = exact_tau(z, r);
  const float below = exp2f(-(alpha - 1.0f) * log2f((float)n));
  float ref = top, lo = -1.0f, tau = -1.0f, hi = -below;
  if (start == 0) {
    vector<float> groups;
    for (int i = 0; i + 8 <= n; i += 8) groups.push_back(*std::max_element(&z[i], &z[i] + 8));
    lo = tau = fminf(fmaxf(-1.0f, (float)exact_tau(groups, r) - 4e-6f), hi);
  } else if (start == 2) {
    ref = *std::max_element(y.begin(), y.begin() + n / 4);
    hi = INFINITY;
    const double off = 0.05 * normal(rng) * -want;
    tau = fmaxf((float)(want + off + ((double)top - ref)), -1.0f);
  }
  vector<float> w(n);
  for (int i = 0; i < n; ++i) w[i] = y[i] - ref;
  SeqSearch<AM> s{tau, lo, hi, (float)n, 0.f, 0.f, 0.f, false, false};
  int sweeps = 0;
  bool done = false;
  while (!done && sweeps < 48) {
    const SeqSums q = sums_at(sweeps == 0 ? w : z, s.tau, r);
    if (sweeps == 0 && start == 2) {  // as the kernel goes on to the row's largest score
      const float up = top - ref;
      s.tau -= up;
      s.lo = fmaxf(s.lo - up, -1.0f);
      s.hi = -below;
    }
    done = s.step(q, r, sweeps == 0 && (AM == 1 || AM == 3));
    ++sweeps;
  }
  seen.sweeps += sweeps;
  ++seen.rows;
  seen.most = std::max(seen.most, sweeps);
  seen.worst = std::max(seen.worst, fabs((double)s.tau - want));
}

int main() {
  const float alphas[] = {1.1f, 1.25f, 1.4f, 1.5f, 1.7f, 1.8f, 1.9f, 1.95f, 1.99f, 2.0f};
  double mean15[3] = {0, 0, 0}, mean2[3] = {0, 0, 0};
  long rows = 0;
  bool good = true;
  printf("ok so far\n");  // (the line by line report follows)
  for (float alpha : alphas)
    for (int start = 0; start < 3; ++start) {
      Seen seen;
      for (float deviation : {0.3f, 1.0f, 5.0f, 15.0f, 40.0f, 1000.0f})
        for (int cluster : {1, 1, 8, 290})
          for (int k = 0; k < 40; ++k) {
            const int n = k % 8 == 0 ? 1500 : (k % 8 == 1 ? 17 : 300);
            if (alpha == 1.5f) row<1>(alpha, n, cluster, deviation, start, seen);
            else if (alpha == 2.0f) row<2>(alpha, n, cluster, deviation, start, seen);
            else if (alpha == 1.25f) row<3>(alpha, n, cluster, deviation, start, seen);
            else row<0>(alpha, n, cluster, deviation, start, seen);
          }
      const double mean = seen.sweeps / seen.rows;
      printf("alpha %.2f start %d: %.2f sweeps a row, at most %d, threshold within %.1e\n", alpha, start, mean, seen.most, seen.worst);
      if (alpha == 1.5f) mean15[start] = mean;
      if (alpha == 2.0f) mean2[start] = mean;
      rows += seen.rows;
      good = good && seen.worst <= 0x1p-19 + 0x1p-22 && seen.most < 24;
    }
  for (int start = 0; start < 3; ++start) good = good && mean2[start] <= 1.5 * mean15[start];
  printf("%s %ld rows\n", good ? "ok" : "failed:", rows);
  return good ? 0 : 1;
}
