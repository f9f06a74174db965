// Whether written and read rows meet, under sanitizers: small random layouts against every byte of them marked.
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

static bool marked(const RowSet& x, std::set<long long>* rows) {  // the first bytes of 4-byte units; false: one twice
  bool apart = true;
  for (long long i = 0; i < x.n[0]; ++i)
    for (long long j = 0; j < x.n[1]; ++j)
      for (long long k = 0; k < x.n[2]; ++k)
        for (long long e = 0; e < x.row; e += 4)
          apart = rows->insert((long long)((const char*)x.at - memory) + i * x.s[0] + j * x.s[1] + k * x.s[2] + e).second && apart;
  return apart;
}

// a part of a dense tensor of up to three axes in any order
static RowSet part(long long (&full)[3], int (&order)[3], long long row_full) {
  RowSet x;
  long long s = row_full;
  for (int k = 2; k >= 0; --k) {
    x.s[order[k]] = s;
    s *= full[order[k]];
  }
  long long at = 0;
  x.row = row_full == 8 && rnd() % 2 ? 4 : row_full;
  if (x.row < row_full) at += 4 * (rnd() % 2);
  for (int k = 0; k < 3; ++k) {
    const long long first = rnd() % full[k];
    x.n[k] = 1 + rnd() % (full[k] - first);
    at += first * x.s[k];
  }
  x.at = memory + at;
  return x;
}

int main() {
  long meet = 0, apart = 0, seen = 0;
  for (; seen < 60000; ++seen) {
    long long full[3] = {1 + rnd() % 4, 1 + rnd() % 4, 1 + rnd() % 3};
    int order[3] = {0, 1, 2};
    std::swap(order[rnd() % 3], order[rnd() % 3]);
    const long long row = rnd() % 2 ? 8 : 4;
    RowSet x = part(full, order, row), y = part(full, order, row);
    std::set<long long> mx, my;
    const bool alone = marked(x, &mx);
    marked(y, &my);
    if (!alone || !rows_apart(x)) return printf("failed: parts of tensors are apart\n"), 1;
    bool truth = false;
    for (long long e : my) truth = truth || mx.count(e) != 0;
    const bool said = rows_meet(x, y);
    const bool exact = x.row == y.row && y.n[0] <= x.n[0] && y.n[1] <= x.n[1] && y.n[2] <= x.n[2];
    if (truth && !said) return printf("failed: they meet\n"), 1;
    if (exact && said != truth) return printf("failed: they do not meet\n"), 1;
    if (same_rows(x, y) && !truth) return printf("failed: the same rows\n"), 1;
    (truth ? meet : apart)++;
    // any strides: what is said to be apart is
    for (int k = 0; k < 3; ++k) x.s[k] = 4 * (rnd() % 12);
    mx.clear();
    if (rows_apart(x) && !marked(x, &mx)) return printf("failed: rows on top of each other\n"), 1;
    mx.clear();
    marked(x, &mx);
    truth = false;
    for (long long e : my) truth = truth || mx.count(e) != 0;
    if (rows_apart(x) && truth && !rows_meet(x, y)) return printf("failed: they meet, other strides\n"), 1;
  }
  // offsets that pass 64 bits
  RowSet far{memory, {1ll << 26, 4096, 1}, {1ll << 42, 1ll << 42, 0}, 128};
  if (rows_apart(far) || rows_meet(RowSet{memory, {4, 1, 1}, {256, 0, 0}, 128}, far) == false) return printf("failed: far\n"), 1;
  if (!rows_apart(RowSet{nullptr, {4, 4, 4}, {0, 0, 0}, 4}) || rows_meet(far, RowSet{nullptr, {1, 1, 1}, {0, 0, 0}, 4})) return printf("failed: nothing\n"), 1;
  printf("ok %ld %ld\n", meet, apart);
  return meet > 1000 && apart > 1000 ? 0 : 1;
}
