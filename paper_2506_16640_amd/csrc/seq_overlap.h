// Whether what a serving call writes meets what it reads, or itself.  Plain C++, no HIP types.
#pragma once
#include <stdint.h>

#include <utility>

namespace entmax {

// Rows of `row` bytes at `at` + i0 s[0] + i1 s[1] + i2 s[2], i_k in 0 .. n[k] - 1 (strides in bytes, not negative)
struct RowSet {
  const void* at;
  long long n[3], s[3];
  long long row;
  bool empty() const { return at == nullptr || n[0] <= 0 || n[1] <= 0 || n[2] <= 0; }
  __int128 extent() const {  // bytes from the first to the end of the last row
    __int128 e = row;
    for (int k = 0; k < 3; ++k) e += (__int128)(n[k] - 1) * s[k];
    return e;
  }
  // the order of the axes from the largest stride to the smallest; those of length one last
  void order(int (&o)[3]) const {
    for (int k = 0; k < 3; ++k) o[k] = k;
    auto key = [&](int k) { return n[k] > 1 ? s[k] : -1; };
    for (int a = 0; a < 2; ++a)
      for (int b = 0; b < 2 - a; ++b)
        if (key(o[b]) < key(o[b + 1])) std::swap(o[b], o[b + 1]);
  }
};

// No two rows meet: every axis steps over all that the axes of smaller strides reach.  (Layouts of tensors and of their slices and permutations do; strides that
// interleave without meeting are counted as meeting.)
inline bool rows_apart(const RowSet& x) {
  if (x.empty()) return true;
  int o[3];
  x.order(o);
  __int128 reach = x.row;
  for (int k = 2; k >= 0; --k) {
    if (x.n[o[k]] <= 1) continue;
    if (x.s[o[k]] < reach) return false;
    reach += (__int128)(x.n[o[k]] - 1) * x.s[o[k]];
  }
  return true;
}

// Whether a row of x (from axis order o[k] on) meets the bytes lo .. hi - 1, counted from x's first.  Rows that are not apart: taken as meeting.
inline bool rows_reach(const RowSet& x, const int (&o)[3], int k, __int128 lo, __int128 hi) {
  if (k == 3 || x.n[o[k]] <= 1) return lo < x.row && hi > 0;
  const __int128 s = x.s[o[k]];
  __int128 inner = x.row;
  for (int e = k + 1; e < 3; ++e) inner += x.n[o[e]] > 1 ? (__int128)(x.n[o[e]] - 1) * x.s[o[e]] : 0;
  if (s < inner) return true;
  // the blocks i s .. i s + inner - 1 that overlap the bytes; of three in a row the middle one begins inside them
  __int128 first = lo < inner ? 0 : (lo - inner) / s + 1, last = hi <= 0 ? -1 : (hi - 1) / s;
  if (last > x.n[o[k]] - 1) last = x.n[o[k]] - 1;
  if (last - first >= 2) return true;
  for (__int128 i = first; i <= last; ++i)
    if (rows_reach(x, o, k + 1, lo - i * s, hi - i * s)) return true;
  return false;
}

// Whether rows of x meet rows of out, whose own are apart.  Exact where the two have the same strides (parts of one tensor) and x is no longer than out along
// any axis; else they are taken as meeting unless one's rows leave free the whole range of memory of the other's.
inline bool rows_meet(const RowSet& out, const RowSet& x) {
  if (out.empty() || x.empty()) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out.at), b = reinterpret_cast<uintptr_t>(x.at);
  if ((__int128)a + out.extent() <= (__int128)b || (__int128)b + x.extent() <= (__int128)a) return false;
  bool alike = x.row == out.row;
  for (int k = 0; k < 3; ++k) alike = alike && x.n[k] <= out.n[k] && (x.n[k] <= 1 || x.s[k] == out.s[k]);
  if (!alike) {
    int ox[3], oo[3];
    x.order(ox);
    out.order(oo);
    const __int128 from = (__int128)a - (__int128)b;
    return rows_reach(x, ox, 0, from, from + out.extent()) && rows_reach(out, oo, 0, -from, -from + x.extent());
  }
  int o[3];
  out.order(o);
  // axis by axis from the largest stride: out's row i and x's row j meet if what is left of their distance is shorter than a row; the axes further in reach
  // less than one stride, so that i - j is one of the two numbers next to distance / stride
  struct Left {
    const RowSet &out, &x;
    const int (&o)[3];
    bool meets(int k, __int128 d) const {
      if (k == 3 || out.n[o[k]] <= 1) return d < out.row && d > -(__int128)out.row;
      const __int128 s = out.s[o[k]];
      const __int128 q = d / s - (d % s < 0 ? 1 : 0);
      for (__int128 m = q; m <= q + 1; ++m)
        if (m > -(__int128)x.n[o[k]] && m < out.n[o[k]] && meets(k + 1, d - m * s)) return true;
      return false;
    }
  };
  return Left{out, x, o}.meets(0, (__int128)b - (__int128)a);
}

// The very same rows
inline bool same_rows(const RowSet& x, const RowSet& y) {
  if (x.at != y.at || x.row != y.row) return false;
  for (int k = 0; k < 3; ++k)
    if (x.n[k] != y.n[k] || (x.n[k] > 1 && x.s[k] != y.s[k])) return false;
  return true;
}

}  // namespace entmax
