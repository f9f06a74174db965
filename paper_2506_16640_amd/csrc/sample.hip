// Sampling of tokens from logits: temperature, top-k, top-p, min-p and the token that a given random number falls on.  With x a row's logits, m the
// largest and w = exp((x - m) / temperature), every filter keeps the first tokens of the row's falling order (x, then lower index first), so that
// what is left is "rank >= cut" for a cut that is found without sorting the row:
//   sample_slices_kernel   a workgroup per slice of a row: its largest logit, its sum of w, and, for rows with top-k or top-p, how many tokens
//                          (top-k) or how much w (top-p) lie in each of 256 bins of equal width below its largest.  Bins lie on one
//                          grid of logits, so that those of a row's slices can be added up.
//   sample_bracket_kernel  the row's bins, and with them the bin in which the filter's cut must lie: tokens above it are surely kept and only their w
//                          is summed, tokens below are dropped, those of the bin are listed
//   sample_pick_kernel     a workgroup per row: the cut by radix selection over the list (ranks are distinct numbers), the slice that the random number
//                          falls into, and the token in it
// A token is right or wrong, and with 10^5 tokens to a row sums of 32 bits would put one row in a hundred on the neighbour of the right one: w and all sums
// are of 64 bits.  Sums that atomics make are sums of integers (w in steps of a power of two), the others are formed in a fixed order: the same call gives the same tokens.
// Bound: one read of the logits, and 64-bit exponentials.
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "common.hip.h"
#include "sample_layout.h"

using namespace entmax;

namespace {

typedef unsigned long long u64;

struct SliceStat {
  double sum;   // of w relative to the slice's own largest logit
  float top;
  int arg;      // its lowest index
  int finite;   // tokens that can be drawn
  int pad;
};
struct SliceKept {
  double all, sum;  // w of the tokens that are surely left by top-k and top-p; of those among them that min-p leaves
  int listed, pad;
};
static_assert(sizeof(SliceStat) == kSampleStatBytes && sizeof(SliceKept) == kSampleStatBytes, "as in make_sample_layout()");

struct SampleArgs {
  const void* logits;
  const float *uniform, *temperature, *top_p, *min_p;
  const int* top_k;
  int* token;
  float* logprob;
  int rows, vocab, nslices;
  long long stride;
  SliceStat* stat;
  float* hist;
  SliceKept* kept;
  uint16_t* cand;
};

// What a row asks for.
struct RowAsk {
  bool greedy, has_k, has_p, has_m;
  int k;
  double inv, p, f, grid;
  __device__ __forceinline__ void init(const SampleArgs& A, int row) {
    auto nan = [](float x) { return (opaque_bits(x) & 0x7fffffffu) > 0x7f800000u; };
    const float t = A.temperature ? A.temperature[row] : 1.f;
    greedy = nan(t) || !(t > 0.f);
    inv = greedy ? 1.0 : 1.0 / (double)t;
    k = A.top_k ? A.top_k[row] : 0;
    has_k = k > 0 && k < A.vocab;
    const float pp = A.top_p ? A.top_p[row] : 1.f, mm = A.min_p ? A.min_p[row] : 0.f;
    has_p = !nan(pp) && pp < 1.f;
    p = has_p ? fmax((double)pp, 0.0) : 1.0;
    has_m = !nan(mm) && mm > 0.f;
    f = has_m ? fmin((double)mm, 1.0) : 0.0;
    // Bins of a twelfth of the temperature: 256 of them reach down to 6e-10 of the largest w, and one holds a few per cent of the tokens of a flat
    // row at most.  Not less than a twelfth of a logit, for top-k at low temperatures.
    grid = greedy ? 0.0 : fmin(12.0 * inv, 12.0);
  }
  __device__ __forceinline__ double weight(float x, float m) const {
    if (x == m) return x == -kInf ? 0.0 : 1.0;  // (m may be infinite)
    if (x == -kInf || m == kInf) return 0.0;
    return exp(((double)x - (double)m) * inv);
  }
  __device__ __forceinline__ int cell(float x) const {
    if (x == kInf) return 1 << 29;
    if (x == -kInf) return -(1 << 29);
    return (int)fmax(fmin(floor((double)x * grid), (double)(1 << 29)), -(double)(1 << 29));
  }
};

// Falling order of logits, and of equal ones by index: larger numbers first.
template <typename T>
struct Rank {
  static constexpr int kBits = 22 + 8 * (int)sizeof(T);
  static __device__ __forceinline__ u64 of(float x, int index) {
    uint32_t b = __float_as_uint(x);
    if (b == 0x80000000u) b = 0u;  // (the two zeros are equal)
    b = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    if (sizeof(T) == 2) b >>= 16;
    return (u64)b << 22 | (u64)(kSampleMostVocab - 1 - index);
  }
};

constexpr int kSampleThreads = 1024;

// A row's slice: thread t has the 16-byte chunks t, t + NT, ..; the slices' addresses are round, so that slice 0 may begin in front of the row.
template <typename T, int NCH>
struct Slice {
  static constexpr int NT = kSampleThreads;
  static constexpr int E = 16 / (int)sizeof(T), N = NCH * E, kSize = NT * N;
  const T* row;
  int vocab, from;  // index of the slice's first place
  __device__ __forceinline__ void init(const SampleArgs& A, int r, int slice) {
    row = reinterpret_cast<const T*>(A.logits) + (long long)r * A.stride;
    vocab = A.vocab;
    from = slice * kSize - (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
  }
  __device__ __forceinline__ int index(int c, int e) const { return from + (c * NT + (int)threadIdx.x) * E + e; }
  static __device__ __forceinline__ float clean(float x) { return (opaque_bits(x) & 0x7fffffffu) > 0x7f800000u ? -kInf : x; }
  static __device__ __forceinline__ float value(T x) {
    if constexpr (sizeof(T) == 2)
      return clean(__uint_as_float((uint32_t)x.bits << 16));
    else
      return clean(x);
  }
  __device__ __forceinline__ float at(int i) const { return value(row[i]); }
  __device__ __forceinline__ void load_chunk(int c, float* x) const {
    const int i0 = index(c, 0);
    if (i0 >= 0 && i0 + E <= vocab) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(row + i0);
#pragma unroll
      for (int e = 0; e < E; ++e)
        x[e] = clean(__uint_as_float(sizeof(T) == 4 ? v[e] : ((e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16)));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = i0 + e >= 0 && i0 + e < vocab ? value(row[i0 + e]) : -kInf;
    }
  }
  __device__ __forceinline__ void load(float (&x)[N]) const {
#pragma unroll
    for (int c = 0; c < NCH; ++c) load_chunk(c, x + c * E);
  }
};

// Sums, largest values over the workgroup, in a fixed order; buf: a number per wave.  (Two barriers.)
template <int NT, typename V, class Op>
__device__ __forceinline__ V reduce(V x, V* buf, Op op) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x = op(x, __shfl_xor(x, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
  __syncthreads();
  V r = buf[threadIdx.x & (NT / 64 - 1)];
#pragma unroll
  for (int off = NT / 128; off >= 1; off >>= 1) r = op(r, __shfl_xor(r, off));
  return r;
}
struct Add {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a + b;
  }
};
struct Most {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a > b ? a : b;
  }
};
struct Least {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a < b ? a : b;
  }
};

// Sums over the threads up to and with this one.
template <int NT>
__device__ __forceinline__ double scan(double x, double* buf, double& total) {
  constexpr int NW = NT / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double y = __shfl_up(x, off);
    if (lane >= off) x += y;
  }
  __syncthreads();
  if (lane == 63) buf[wave] = x;
  __syncthreads();
  double w = buf[lane & (NW - 1)];
#pragma unroll
  for (int off = 1; off < NW; off <<= 1) {
    const double y = __shfl_up(w, off);
    if ((lane & (NW - 1)) >= off) w += y;
  }
  total = __shfl(w, NW - 1);
  const double before = __shfl(w, wave > 0 ? wave - 1 : 0);
  return x + (wave > 0 ? before : 0.0);
}

// w in whole steps of 2^-44: a slice's sum stays below 2^58
constexpr double kSliceSteps = 17592186044416.0;

template <typename T, int NCH>
__global__ __launch_bounds__(kSampleThreads) void sample_slices_kernel(SampleArgs A) {
  constexpr int NT = kSampleThreads;
  using S = Slice<T, NCH>;
  __shared__ u64 buf[NT / 64];
  __shared__ u64 bins[kSampleBins];
  const int row = blockIdx.x / A.nslices, slice = blockIdx.x - row * A.nslices, tid = threadIdx.x;
  S sl;
  sl.init(A, row, slice);
  float x[S::N];
  sl.load(x);
  RowAsk ask;
  ask.init(A, row);
  u64 best = 0;
  int finite = 0;
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float v = x[c * S::E + e];
      if (v == -kInf) continue;
      ++finite;
      const u64 r = Rank<float>::of(v, sl.index(c, e));
      best = r > best ? r : best;
    }
  best = reduce<NT>(best, buf, Most());
  finite = reduce<NT>(finite, reinterpret_cast<int*>(buf), Add());
  float top = -kInf;
  if (best) {
    const uint32_t b = (uint32_t)(best >> 22);
    top = __uint_as_float((b & 0x80000000u) ? b & 0x7fffffffu : ~b);
  }
  const long long at = (long long)row * A.nslices + slice;
  double sum = 0.0;
  if (!ask.greedy && best) {  // (uniform)
    const bool binned = ask.has_k || ask.has_p;
    if (binned) {
      if (tid < kSampleBins) bins[tid] = 0;
      __syncthreads();
    }
    const int cell = ask.cell(top);
#pragma unroll
    for (int e = 0; e < S::N; ++e) {
      if (x[e] == -kInf) continue;
      const double w = ask.has_k ? 0.0 : ask.weight(x[e], top);
      sum += w;
      const int b = binned ? cell - ask.cell(x[e]) : kSampleBins;
      if (b < kSampleBins - 1) atomicAdd(&bins[b], ask.has_k ? 1ull : (u64)(w * kSliceSteps + 0.5));
    }
    sum = reduce<NT>(sum, reinterpret_cast<double*>(buf), Add());
    if (binned && tid < kSampleBins) A.hist[at * kSampleBins + tid] = ask.has_k ? (float)bins[tid] : (float)((double)bins[tid] / kSliceSteps);
  }
  if (tid == 0) A.stat[at] = SliceStat{sum, top, best ? kSampleMostVocab - 1 - (int)(best & (kSampleMostVocab - 1)) : -1, finite, 0};
}

// What the slices say of a row, the same in every thread.
struct RowStat {
  float top;
  int finite;
  double sum;  // of w, relative to the row's largest (rows without top-k)
};
template <int NT>
__device__ __forceinline__ RowStat row_stat(const SampleArgs& A, const RowAsk& ask, int row, u64* buf) {
  const SliceStat* st = A.stat + (long long)row * A.nslices;
  float top = -kInf;
  int finite = 0;
  for (int s = threadIdx.x; s < A.nslices; s += NT) {
    top = fmaxf(top, st[s].top);
    finite += st[s].finite;
  }
  RowStat r;
  r.top = reduce<NT>(top, reinterpret_cast<float*>(buf), Most());
  r.finite = reduce<NT>(finite, reinterpret_cast<int*>(buf), Add());
  double sum = 0.0;
  if (!ask.greedy && !ask.has_k)
    for (int s = threadIdx.x; s < A.nslices; s += NT) sum += st[s].sum * ask.weight(st[s].top, r.top);
  r.sum = reduce<NT>(sum, reinterpret_cast<double*>(buf), Add());
  return r;
}

template <typename T, int NCH>
__global__ __launch_bounds__(kSampleThreads) void sample_bracket_kernel(SampleArgs A) {
  constexpr int NT = kSampleThreads;
  using S = Slice<T, NCH>;
  __shared__ u64 buf[NT / 64];
  __shared__ int listed;
  const int row = blockIdx.x / A.nslices, slice = blockIdx.x - row * A.nslices, tid = threadIdx.x;
  RowAsk ask;
  ask.init(A, row);
  if (ask.greedy || !(ask.has_k || ask.has_p || ask.has_m)) return;
  S sl;
  sl.init(A, row, slice);
  float x[S::N];
  sl.load(x);
  const RowStat r = row_stat<NT>(A, ask, row, buf);
  const int cell = ask.cell(r.top);
  int b0 = kSampleBins, b1 = -1;  // tokens in bins below b0 are surely kept, those of b0 .. b1 listed
  if (ask.has_k || ask.has_p) {
    // the row's bins: thread b adds up its bin over the slices, in their order; what lies in no bin is in the last
    const SliceStat* st = A.stat + (long long)row * A.nslices;
    const float* hist = A.hist + (long long)row * A.nslices * kSampleBins;
    double mine = 0.0;
    if (tid < kSampleBins - 1)
      for (int s = 0; s < A.nslices; ++s) {
        const float top = st[s].top;
        if (top == -kInf) continue;
        const int b = tid - (cell - ask.cell(top));
        if (b >= 0) mine += (double)hist[s * kSampleBins + b] * (ask.has_k ? 1.0 : ask.weight(top, r.top));
      }
    double all;
    const double upto = scan<NT>(mine, reinterpret_cast<double*>(buf), all);
    // where the sum reaches what is to be kept.  Sums of w: a little less and a little more of it, for the rounding of the bins
    const double least = ask.has_k ? (double)ask.k : ask.p * r.sum * (1.0 - 1e-5), most = ask.has_k ? (double)ask.k : ask.p * r.sum * (1.0 + 1e-5);
    const int n0 = __syncthreads_count(tid < kSampleBins - 1 && upto < least), n1 = __syncthreads_count(tid < kSampleBins - 1 && upto < most);
    b0 = ask.has_k ? 0 : n0;  // (what top-p takes its part of is the w of top-k's tokens: they are all listed)
    b1 = n1;
  }
  if (tid == 0) listed = 0;
  __syncthreads();
  double sum_all = 0.0, sum = 0.0;
  const long long at = (long long)row * A.nslices + slice;
  uint16_t* cand = A.cand + at * S::kSize;
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float v = x[c * S::E + e];
      const int b = v == -kInf ? kSampleBins : min(cell - ask.cell(v), kSampleBins - 1);
      if (b < b0) {
        const double w = ask.weight(v, r.top);
        sum_all += w;
        sum += w >= ask.f ? w : 0.0;
      } else if (b <= b1) {
        cand[atomicAdd(&listed, 1)] = (uint16_t)((c * NT + tid) * S::E + e);
      }
    }
  sum_all = reduce<NT>(sum_all, reinterpret_cast<double*>(buf), Add());
  sum = reduce<NT>(sum, reinterpret_cast<double*>(buf), Add());
  if (tid == 0) A.kept[at] = SliceKept{sum_all, sum, listed, 0};
}

constexpr int kPickList = 6144;    // listed tokens that stay in LDS; longer lists are looked up again for every pass

struct PickLds {
  u64 buf[kSampleThreads / 64];
  u64 bins[kSampleBins];
  u64 rank[kPickList];
  u64 steps[kPickList];   // w in steps
  int cut_bin;
  u64 before;
};

template <typename T, int NCH>
__global__ __launch_bounds__(kSampleThreads) void sample_pick_kernel(SampleArgs A, int filtered) {
  constexpr int NT = kSampleThreads;
  using S = Slice<T, NCH>;
  __shared__ PickLds lds;
  const int row = blockIdx.x, tid = threadIdx.x;
  RowAsk ask;
  ask.init(A, row);
  const RowStat r = row_stat<NT>(A, ask, row, lds.buf);
  const long long at = (long long)row * A.nslices;
  if (r.finite == 0) {
    if (tid == 0) {
      A.token[row] = -1;
      if (A.logprob) A.logprob[row] = -kInf;
    }
    return;
  }
  if (ask.greedy) {
    int arg = kSampleMostVocab;
    for (int s = tid; s < A.nslices; s += NT)
      if (A.stat[at + s].top == r.top) arg = min(arg, A.stat[at + s].arg);
    arg = reduce<NT>(arg, reinterpret_cast<int*>(lds.buf), Least());
    if (tid == 0) {
      A.token[row] = arg;
      if (A.logprob) A.logprob[row] = 0.f;
    }
    return;
  }
  const bool cuts = filtered && (ask.has_k || ask.has_p), sums = filtered && (cuts || ask.has_m);
  u64 cut = 0;  // tokens of this rank and above are left by top-k and top-p
  int listed = 0;
  double steps = 1.0;  // steps of w that make 1
  // every listed token: fn(rank, w in steps)
  auto each = [&](auto fn) {
    if (listed <= kPickList) {
      for (int i = tid; i < listed; i += NT) fn(lds.rank[i], lds.steps[i]);
      return;
    }
    for (int s = 0; s < A.nslices; ++s) {
      S sl;
      sl.init(A, row, s);
      const int n = A.kept[at + s].listed;
      const uint16_t* cand = A.cand + (at + s) * S::kSize;
      for (int i = tid; i < n; i += NT) {
        const int j = sl.from + cand[i];
        const float x = sl.at(j);
        fn(Rank<T>::of(x, j), (u64)(ask.weight(x, r.top) * steps + 0.5));
      }
    }
  };
  // Of the listed tokens of rank >= least and with an amount: the rank of the last one in falling order before which the amounts add up to less than
  // `target` (at least 1).
  auto select = [&](u64 target, u64 least, auto amount) {
    u64 lo = ~0ull, hi = 0;
    each([&](u64 k, u64 w) {
      if (k < least || amount(w) == 0) return;
      lo = k < lo ? k : lo;
      hi = k > hi ? k : hi;
    });
    lo = reduce<NT>(lo, lds.buf, Least());
    hi = reduce<NT>(hi, lds.buf, Most());
    if (lo > hi) return least;  // (none has)
    u64 before = 0;  // amount of the ranks above hi
    while (lo < hi) {  // the rank is in lo .. hi, which agree above bit `shift + 8`
      const int shift = max(0, 64 - __clzll((long long)(lo ^ hi)) - 8);
      __syncthreads();
      if (tid < kSampleBins) lds.bins[tid] = 0;
      __syncthreads();
      each([&](u64 k, u64 w) {
        if (k >= lo && k <= hi) atomicAdd(&lds.bins[(k >> shift) & 255], amount(w));
      });
      __syncthreads();
      // bins from the highest down: the last one with something in it, before which the sum is below the target
      if (tid < 64) {
        u64 v[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = lds.bins[255 - 4 * tid - j];
          mine += v[j];
        }
        u64 upto = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const u64 y = __shfl_up(upto, off);
          if (tid >= off) upto += y;
        }
        u64 sum = before + upto - mine, b_before = 0;
        int b = -1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (v[j] != 0 && sum < target) {
            b = 255 - 4 * tid - j;
            b_before = sum;
          }
          sum += v[j];
        }
        const u64 lanes = __ballot(b >= 0);
        const int lane = 63 - __clzll((long long)lanes);
        if (tid == lane) {
          lds.cut_bin = b;
          lds.before = b_before;
        }
      }
      __syncthreads();
      const u64 base = ((lo >> shift) & ~255ull) + (u64)lds.cut_bin;
      before = lds.before;
      // the ranks of that bin, closed in on
      const u64 from = max(lo, base << shift), to = min(hi, ((base + 1) << shift) - 1);
      u64 l = ~0ull, h = 0;
      each([&](u64 k, u64 w) {
        if (k < from || k > to || amount(w) == 0) return;
        l = k < l ? k : l;
        h = k > h ? k : h;
      });
      lo = reduce<NT>(l, lds.buf, Least());
      hi = reduce<NT>(h, lds.buf, Most());
    }
    return lo;
  };
  if (cuts) {
    int n = 0;
    for (int s = tid; s < A.nslices; s += NT) n += A.kept[at + s].listed;
    listed = reduce<NT>(n, reinterpret_cast<int*>(lds.buf), Add());
    steps = exp2((double)(62 - (32 - __clz(listed | 1))));  // (w <= 1: sums stay below 2^63)
    if (listed <= kPickList) {
      int first = 0;
      for (int s = 0; s < A.nslices; ++s) {
        S sl;
        sl.init(A, row, s);
        const int m = A.kept[at + s].listed;
        const uint16_t* cand = A.cand + (at + s) * S::kSize;
        for (int i = tid; i < m; i += NT) {
          const int j = sl.from + cand[i];
          const float x = sl.at(j);
          lds.rank[first + i] = Rank<T>::of(x, j);
          lds.steps[first + i] = (u64)(ask.weight(x, r.top) * steps + 0.5);
        }
        first += m;
      }
      __syncthreads();
    }
    if (ask.has_k && listed >= ask.k) cut = select((u64)ask.k, 0, [](u64) { return 1ull; });
    if (ask.has_p) {
      double total = r.sum, before = 0.0;  // of what top-k leaves, and of what is surely kept
      if (ask.has_k) {
        u64 t = 0;
        each([&](u64 k, u64 w) { t += k >= cut ? w : 0; });
        total = (double)reduce<NT>(t, lds.buf, Add()) / steps;
      } else {
        double b = 0.0;
        for (int s = tid; s < A.nslices; s += NT) b += A.kept[at + s].all;
        before = reduce<NT>(b, reinterpret_cast<double*>(lds.buf), Add());
      }
      // (whole steps before a token are fewer than the target's if they are fewer than it rounded up; the first token stays)
      const double target = ceil((ask.p * total - before) * steps);
      if (listed > 0) cut = max(cut, select(target >= 1.0 ? (u64)target : 1ull, cut, [](u64 w) { return w; }));
    }
  }
  // ---------------------------------------------------------------- the slice that the random number falls into
  const float un = A.uniform[row];
  const double u = (opaque_bits(un) & 0x7fffffffu) > 0x7f800000u ? 0.0 : fmin(fmax((double)un, 0.0), 1.0);
  const int wave = tid >> 6, lane = tid & 63;
  // w of slice s that is left; all lanes of a wave together
  auto slice_sum = [&](int s) {
    if (!sums) return A.stat[at + s].sum * ask.weight(A.stat[at + s].top, r.top);
    double sum = A.kept[at + s].sum;
    if (cuts) {
      u64 t = 0;
      S sl;
      sl.init(A, row, s);
      const int n = A.kept[at + s].listed;
      const uint16_t* cand = A.cand + (at + s) * S::kSize;
      for (int i = lane; i < n; i += 64) {
        const int j = sl.from + cand[i];
        const float x = sl.at(j);
        const double w = ask.weight(x, r.top);
        if (Rank<T>::of(x, j) >= cut && w >= ask.f) t += (u64)(w * steps + 0.5);
      }
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) t += __shfl_xor(t, off);
      sum += (double)t / steps;
    }
    return sum;
  };
  __shared__ double slice_sums[kSampleMostVocab / kSampleLargeSlice + 1];
  __shared__ int chosen, first, found;
  __shared__ double left;  // of the random number's share in the chosen slice
  __shared__ double all;
  for (int s = wave; s < A.nslices; s += NT / 64) {
    const double x = slice_sum(s);
    if (lane == 0) slice_sums[s] = x;
  }
  __syncthreads();
  if (tid == 0) {
    double total = 0.0;
    for (int s = 0; s < A.nslices; ++s) total += slice_sums[s];
    const double want = u * total;
    double sum = 0.0;
    int pick = -1;
    for (int s = 0; s < A.nslices; ++s) {
      if (slice_sums[s] > 0.0) {
        pick = s;
        left = want - sum;
        if (sum + slice_sums[s] > want) break;
      }
      sum += slice_sums[s];
    }
    chosen = pick;
    all = total;
    found = -1;
    first = NT;
  }
  __syncthreads();
  // ---------------------------------------------------------------- the token in it
  S sl;
  sl.init(A, row, chosen);
  const double want = left;
  double before = 0.0;
  int last = -1;  // the last token of this thread that is left
  for (int c = 0; c < NCH; ++c) {
    float x[S::E];
    sl.load_chunk(c, x);
    double w[S::E], sum = 0.0;
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      w[e] = ask.weight(x[e], r.top);
      if (!(w[e] >= ask.f) || Rank<T>::of(x[e], sl.index(c, e)) < cut) w[e] = 0.0;
      if (w[e] > 0.0) last = sl.index(c, e);
      sum += w[e];
    }
    double total;
    double upto = before + scan<NT>(sum, reinterpret_cast<double*>(lds.buf), total);
    if (sum > 0.0 && upto > want) atomicMin(&first, tid);
    __syncthreads();
    if (first < NT) {  // (uniform)
      if (tid == first) {
        double t = upto - sum;
        int pick = -1;
        bool over = false;
#pragma unroll
        for (int e = 0; e < S::E; ++e) {
          t += w[e];
          if (w[e] > 0.0 && !over) {
            pick = sl.index(c, e);
            over = t > want;
          }
        }
        found = pick;
      }
      break;
    }
    before += total;
  }
  __syncthreads();
  int token = found;
  if (token < 0) token = reduce<NT>(last, reinterpret_cast<int*>(lds.buf), Most());  // (a sum that rounding left just short)
  if (tid == 0) {
    A.token[row] = token;
    if (A.logprob) A.logprob[row] = token < 0 ? -kInf : (float)log(ask.weight(sl.at(token), r.top) / all);
  }
}

template <typename T, int NCH>
bool launch_sample(const SampleArgs& a, hipStream_t st) {
  static_assert(Slice<T, NCH>::kSize == kSampleSmallSlice || Slice<T, NCH>::kSize == kSampleLargeSlice, "as in sample_slice()");
  const bool filtered = a.top_k || a.top_p || a.min_p;
  const dim3 grid((unsigned)((long long)a.rows * a.nslices));
  hipLaunchKernelGGL((sample_slices_kernel<T, NCH>), grid, dim3(kSampleThreads), 0, st, a);
  if (hipGetLastError() != hipSuccess) return false;
  if (filtered) {
    hipLaunchKernelGGL((sample_bracket_kernel<T, NCH>), grid, dim3(kSampleThreads), 0, st, a);
    if (hipGetLastError() != hipSuccess) return false;
  }
  hipLaunchKernelGGL((sample_pick_kernel<T, NCH>), dim3((unsigned)a.rows), dim3(kSampleThreads), 0, st, a, filtered ? 1 : 0);
  return hipGetLastError() == hipSuccess;
}

inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace

extern "C" {

size_t entmax_sample_workspace_bytes(const entmax_sample_params* p) {
  return check_sample_params(p) == ENTMAX_ATTN_OK ? make_sample_layout(p).total : 0;
}

int entmax_sample(const entmax_sample_params* p, const void* logits, const float* uniform, const float* temperature, const int32_t* top_k,
                  const float* top_p, const float* min_p, int32_t* token, float* logprob, void* workspace, size_t workspace_bytes,
                  void* hip_stream) {
  const int rc = check_sample_params(p);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->rows == 0) return ENTMAX_ATTN_OK;
  if (!logits || !uniform || !token || !workspace) return ENTMAX_ATTN_INVALID_ARG;
  const size_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es != 0 || off4(uniform) || off4(temperature) || off4(top_k) || off4(top_p) || off4(min_p) ||
      off4(token) || off4(logprob) || (reinterpret_cast<uintptr_t>(workspace) & 15u) != 0)
    return ENTMAX_ATTN_MISALIGNED;
  const SampleLayout L = make_sample_layout(p);
  if (workspace_bytes < L.total) return ENTMAX_ATTN_WORKSPACE_TOO_SMALL;
  if (!sample_outputs_apart(p, logits, uniform, temperature, top_k, top_p, min_p, token, logprob, workspace, L.total)) return ENTMAX_ATTN_INVALID_ARG;
  char* ws = reinterpret_cast<char*>(workspace);
  SampleArgs a;
  a.logits = logits;
  a.uniform = uniform;
  a.temperature = temperature;
  a.top_p = top_p;
  a.min_p = min_p;
  a.top_k = top_k;
  a.token = token;
  a.logprob = logprob;
  a.rows = p->rows;
  a.vocab = p->vocab;
  a.nslices = L.nslices;
  a.stride = p->stride;
  a.stat = reinterpret_cast<SliceStat*>(ws + L.off_stat);
  a.hist = reinterpret_cast<float*>(ws + L.off_hist);
  a.kept = reinterpret_cast<SliceKept*>(ws + L.off_kept);
  a.cand = reinterpret_cast<uint16_t*>(ws + L.off_cand);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const bool small = L.slice == kSampleSmallSlice;
  bool ok;
  if (p->dtype == ENTMAX_ATTN_BF16)
    ok = small ? launch_sample<bf16_t, 1>(a, st) : launch_sample<bf16_t, 2>(a, st);
  else
    ok = small ? launch_sample<float, 2>(a, st) : launch_sample<float, 4>(a, st);
  return ok ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // extern "C"
