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

// Whether rows of x meet rows of out, whose own are apart.  Exact where the two have the same strides (parts of one tensor) and x is no longer than out along
// any axis; else they meet if one's range of memory meets the other's.
inline bool rows_meet(const RowSet& out, const RowSet& x) {
  if (out.empty() || x.empty()) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out.at), b = reinterpret_cast<uintptr_t>(x.at);
  if ((__int128)a + out.extent() <= (__int128)b || (__int128)b + x.extent() <= (__int128)a) return false;
  for (int k = 0; k < 3; ++k)
    if (x.row != out.row || x.n[k] > out.n[k] || (x.n[k] > 1 && x.s[k] != out.s[k])) return true;
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
