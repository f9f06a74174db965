// Rows of one tensor in the gaps of another's (other strides), under sanitizers: small random layouts against every byte of them marked.
#include <stdio.h>

#include <set>

#include "seq_overlap.h"

using namespace entmax;

static unsigned long long state = 88172645463325252ull;
static unsigned rnd() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return (unsigned)(state >> 16);
}
static char memory[1 << 16];  // (addresses only)

static void mark(const RowSet& x, std::set<long long>* rows) {
  for (long long i = 0; i < x.n[0]; ++i)
    for (long long j = 0; j < x.n[1]; ++j)
      for (long long k = 0; k < x.n[2]; ++k)
        for (long long e = 0; e < x.row; e += 4) rows->insert((long long)((const char*)x.at - memory) + i * x.s[0] + j * x.s[1] + k * x.s[2] + e);
}
static RowSet any(int gaps) {
  RowSet x;
  x.at = memory + 4 * (rnd() % 60);
  x.row = 4 * (1 + rnd() % 2);
  int order[3] = {0, 1, 2};
  std::swap(order[rnd() % 3], order[rnd() % 3]);
  long long reach = x.row;
  for (int k = 0; k < 3; ++k) {
    const int at = order[k];
    x.n[at] = 1 + rnd() % 4;
    x.s[at] = reach + 4 * (rnd() % gaps);
    reach += (x.n[at] - 1) * x.s[at];
  }
  return x;
}

int main() {
  long meet = 0, apart = 0, free_range = 0;
  for (long seen = 0; seen < 100000; ++seen) {
    const RowSet out = any(12), x = any(seen % 2 ? 1 : 12);
    if (!rows_apart(out) || !rows_apart(x)) return printf("failed: they are apart in themselves\n"), 1;
    std::set<long long> mo, mx;
    mark(out, &mo);
    mark(x, &mx);
    bool truth = false, in_out = false, in_x = false;
    for (long long e : mx) truth = truth || mo.count(e), in_out = in_out || (e >= *mo.begin() && e <= *mo.rbegin());
    for (long long e : mo) in_x = in_x || (e >= *mx.begin() && e <= *mx.rbegin());
    const bool said = rows_meet(out, x);
    if (truth && !said) return printf("failed: they meet\n"), 1;
    // one leaves the other's whole range free (for parts of one tensor the answer is exact and may be no as well)
    if ((!in_out || !in_x) && said) return printf("failed: the range is free\n"), 1;
    if (!in_out || !in_x) ++free_range;
    (truth ? meet : apart)++;
  }
  printf("ok %ld %ld %ld\n", meet, apart, free_range);
  return meet > 1000 && apart > 1000 && free_range > 1000 ? 0 : 1;
}
