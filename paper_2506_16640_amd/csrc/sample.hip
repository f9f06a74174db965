// Sampling of tokens from logits: temperature, top-k, top-p, min-p and the token that a given random number falls on.  With x a row's logits, m the
// largest and w = exp((x - m) / temperature), every filter keeps the first tokens of the row's falling order (x, then lower index first), so that
// what is left is "rank >= cut" for a cut that is found without sorting the row:
//   sample_slices_kernel   a workgroup per slice of a row: its largest logit, its sum of w, and, for rows with top-k or top-p, how many tokens
//                          (top-k) or how much w (top-p) lie in each of 512 bins of equal width below its largest.  Bins lie on one
//                          grid of logits, so that those of a row's slices can be added up.
//   sample_bracket_kernel  the row's bins, and with them the bin in which the filter's cut must lie: tokens above it are surely kept and only their w
//                          is summed, tokens below are dropped, those of the bin are listed
//   sample_pick_kernel     a workgroup per row: the cut by radix selection over the list (ranks are distinct numbers), the slice that the random number
//                          falls into, and the token in it
// A token is right or wrong, and with 10^5 tokens to a row sums of 32 bits would put one row in a hundred on the neighbour of the right one: w and all sums
// are of 64 bits.  Sums that atomics make are sums of integers (w in steps of a power of two), the others are formed in a fixed order: the same call gives the same tokens.
// Bound: one read of the logits and 64-bit exponentials (256 plain rows of 32768 in fp32: 15.5 us of 21, 7 of them reading); with filters, three dependent
// launches of round trips (64 rows of 131072: 16 + 22 + 18 us).
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "common.hip.h"
#include "sample_layout.h"
#include "wave_ops.hip.h"

using namespace entmax;

namespace {

typedef unsigned long long u64;

struct SliceStat {
  double sum;   // of w relative to the slice's own largest logit (rows without top-k)
  float top;
  int arg;      // its lowest index (rows that take the largest logit)
};
struct SliceKept {
  double all, sum;  // w of the tokens that are surely left by top-k and top-p; of those among them that min-p leaves
  int listed, pad;  // tokens that have to be looked at
};
static_assert(sizeof(SliceStat) == kSampleStatBytes && sizeof(SliceKept) == kSampleKeptBytes, "as in make_sample_layout()");

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
  double* blocks;  // [slices][blocks of a slice] w of the tokens of each block, as in SliceKept::sum or SliceStat::sum
  char* cand;   // [slices][tokens of a slice] Listed<T>
};

// What a row asks for.
struct RowAsk {
  bool greedy, has_k, has_p, has_m;
  int k;
  double scale, p, f;  // log2(w) of a logit of 1; top_p, min_p
  float grid;          // bins of a logit of 1
  __device__ __forceinline__ void init(const SampleArgs& A, int row) {
    auto nan = [](float x) { return (opaque_bits(x) & 0x7fffffffu) > 0x7f800000u; };
    const float t = A.temperature ? A.temperature[row] : 1.f;
    greedy = nan(t) || !(t > 0.f);
    const double inv = greedy ? 1.0 : 1.0 / (double)t;
    scale = fmax(inv * 1.4426950408889634, 1e-300);  // (more than zero, so that -infinity stays what it is; 1e-300 of a logit is nothing)
    k = A.top_k ? A.top_k[row] : 0;
    has_k = k > 0 && k < A.vocab;
    const float pp = A.top_p ? A.top_p[row] : 1.f, mm = A.min_p ? A.min_p[row] : 0.f;
    has_p = !nan(pp) && pp < 1.f;
    p = has_p ? fmax((double)pp, 0.0) : 1.0;
    has_m = !nan(mm) && mm > 0.f;
    f = has_m ? fmin((double)mm, 1.0) : 0.0;
    // top-p: bins of 1/32 of the temperature.  512 of them reach down to 1e-7 of the largest w, below which lies nothing that counts (256 of 1/24 of it reached down
    // to 2e-5, and where the cut of 131072 tokens, a few of which stood out, was in none of them, all were listed and the call took 500 us for 50), and the bin
    // of the cut holds a few per cent of the tokens of a flat row at most.  top-k: 1/12 of it, but not less than 1/12 of a logit, for low temperatures.
    grid = greedy ? 0.f : (float)fmin(has_k ? fmin(12.0 * inv, 12.0) : 32.0 * inv, 1e30);
  }
  // 2^t, t <= 0, to 4e-14 of it and 1 for 0: the whole part goes to the exponent; the rest f, at most 1/2, through 1 + f p(f), p interpolating (2^f - 1) / f at the
  // nine zeros of a Chebyshev polynomial.  (From -1100 on: the whole part is one of 32 bits)
  static __device__ __forceinline__ double power(double t) {
    const double k = rint(t), f = t - k;
    double p = 1.0203121172135084e-07;
    p = fma(p, f, 1.3255224874051843e-06);
    p = fma(p, f, 1.5252686845751599e-05);
    p = fma(p, f, 0.00015403455852473414);
    p = fma(p, f, 0.0013333558179043862);
    p = fma(p, f, 0.009618129159402536);
    p = fma(p, f, 0.055504108664760424);
    p = fma(p, f, 0.2402265069581299);
    p = fma(p, f, 0.6931471805599453);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)k);
  }
  // w of a logit x next to the largest, m
  __device__ __forceinline__ double weight(float x, float m) const {
    if (m == kInf || m == -kInf) return x == m && x > 0.f ? 1.0 : 0.0;  // (uniform)
    // (below 2^-1074 all are 0.  Unbounded, t - k would be formed from the product before it is rounded, which beyond 2^53 is a number of any size)
    return power(fmax(((double)x - (double)m) * scale, -1100.0));
  }
  // The logit's place on the row's grid of bins.  (That it never falls as x rises is all that matters: bins of a row's slices are the same ones.  Negative logits
  // are below 0 also where their product is none: edge() could not find the end of those otherwise.)
  __device__ __forceinline__ int cell(float x) const {
    if (x == kInf) return 1 << 29;
    if (x == -kInf) return -(1 << 29);
    return (int)fminf(fmaxf(floorf(x * grid), -(float)(1 << 29)), x < 0.f ? -1.f : (float)(1 << 29));
  }
  // The smallest logit of cell c or above (-inf: all of them are)
  __device__ __forceinline__ float edge(int c) const {
    if (c <= -(1 << 29)) return -kInf;
    if (grid == 0.f) return c < 0 ? -kInf : c == 0 ? 0.f : kInf;
    constexpr float kMost = 3.40282347e38f;  // (the largest finite number: it and its negative may be logits)
    float x = fminf(fmaxf((float)c / grid, -kMost), kMost);
    // (the quotient is rounded, and so are products: a few steps of a float away at most; with a step of zero nothing but infinity is left)
    for (int k = 0; k < 8 && cell(x) >= c && x > -kMost; ++k) x = next(x, -1);
    for (int k = 0; k < 16 && cell(x) < c; ++k) x = next(x, 1);
    return x;
  }
  static __device__ __forceinline__ float next(float x, int way) {  // the neighbour of a finite number (the largest one's: infinity)
    const int b = (int)__float_as_uint(x), order = b < 0 ? (int)(0x80000000u - (uint32_t)b) : b;
    const int n = order + way;
    return __uint_as_float(n < 0 ? 0x80000000u - (uint32_t)n : (uint32_t)n);
  }
};

// Falling order of logits, and of equal ones by index: larger numbers first.
template <typename T>
struct Rank {
  static __device__ __forceinline__ uint32_t key(float x) {
    uint32_t b = __float_as_uint(x);
    if (b == 0x80000000u) b = 0u;  // (the two zeros are equal)
    b = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return sizeof(T) == 2 ? b >> 16 : b;
  }
  static __device__ __forceinline__ u64 of(uint32_t key, int index) { return (u64)key << 22 | (u64)(kSampleMostVocab - 1 - index); }
  static __device__ __forceinline__ u64 of(float x, int index) { return of(key(x), index); }
  static __device__ __forceinline__ float logit(uint32_t key) {
    if (sizeof(T) == 2) key = key << 16 | ((key & 0x8000u) ? 0u : 0xffffu);
    return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
  }
};
// A listed token: key and place in its slice
template <typename T>
struct Listed {
  typedef u64 Word;
  static __device__ __forceinline__ Word pack(uint32_t key, int place) { return (u64)key << 16 | (u64)place; }
  static __device__ __forceinline__ uint32_t key(Word w) { return (uint32_t)(w >> 16); }
  static __device__ __forceinline__ int place(Word w) { return (int)(w & 0xffffu); }
};
template <>
struct Listed<bf16_t> {
  typedef uint32_t Word;
  static __device__ __forceinline__ Word pack(uint32_t key, int place) { return key << 16 | (uint32_t)place; }
  static __device__ __forceinline__ uint32_t key(Word w) { return w >> 16; }
  static __device__ __forceinline__ int place(Word w) { return (int)(w & 0xffffu); }
};

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;

// A row's slice: thread t has the 16-byte chunks t, t + NT, ..; the slices' addresses are round, so that slice 0 may begin in front of the row.
template <typename T, int NCH>
struct Slice {
  static constexpr int NT = kSampleThreads;
  static constexpr int E = 16 / (int)sizeof(T), N = NCH * E, kSize = NT * N;
  static constexpr int kBlock = 64 * E, kBlocks = kSize / kBlock;  // what a wave loads at a time: block c kSampleWaves + wave
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
  __device__ __forceinline__ void load_chunk(int i0, float* x) const {
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
    for (int c = 0; c < NCH; ++c) load_chunk(index(c, 0), x + c * E);
  }
};

// A number below 2^52 as a whole one, by the place where the sum's bits end
__device__ __forceinline__ u64 whole(double x) { return (u64)__double_as_longlong(x + 4503599627370496.0) & 0xfffffffffffffull; }
// The sums of a workgroup's blocks, `part` a thread's w of each of its chunks; returns their sum, the same in every thread.  (Two barriers.)
template <int NCH>
__device__ __forceinline__ double sum_blocks(const double (&part)[NCH], double (&sums)[NCH * kSampleWaves], double* out) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  static_assert(NCH * kSampleWaves <= 64, "a lane each");
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const double x = wave_reduce(part[c], 0.0, Add());
    if (lane == 0) sums[c * kSampleWaves + wave] = x;
  }
  __syncthreads();
  const double x = lane < NCH * kSampleWaves ? sums[lane] : 0.0;
  if (out && wave == 0 && lane < NCH * kSampleWaves) out[lane] = x;
  return wave_reduce(x, 0.0, Add());
}

// What the rounding of w and of sums of them stays far below: numbers that are nearer to each other than this part of them are taken as equal
constexpr double kRounding = 2.3e-13;
// w in whole steps of 2^-44 where slices' bins are added up: a slice's sum stays below 2^58
constexpr double kSliceSteps = 17592186044416.0;

// (two workgroups to a compute unit: at most 64 registers)
template <typename T, int NCH>
__global__ __launch_bounds__(kSampleThreads, 8) void sample_slices_kernel(SampleArgs A) {
  constexpr int NT = kSampleThreads;
  using S = Slice<T, NCH>;
  __shared__ u64 buf[kSampleWaves];
  __shared__ u64 bins[kSampleBins];
  __shared__ double sums[S::kBlocks];
  const int row = blockIdx.x / A.nslices, slice = blockIdx.x - row * A.nslices, tid = threadIdx.x;
  S sl;
  sl.init(A, row, slice);
  float x[S::N];
  sl.load(x);
  RowAsk ask;
  ask.init(A, row);
  const bool binned = !ask.greedy && (ask.has_k || ask.has_p);
  if (binned && tid < kSampleBins) bins[tid] = 0;
  float top = x[0];
#pragma unroll
  for (int e = 1; e < S::N; ++e) top = fmaxf(top, x[e]);
  top = block_reduce<kSampleWaves>(top, -kInf, reinterpret_cast<float*>(buf), Most());
  const long long at = (long long)row * A.nslices + slice;
  double sum = 0.0;
  int arg = kSampleMostVocab;
  if (ask.greedy) {  // (uniform, like the other ways here)
#pragma unroll
    for (int c = NCH - 1; c >= 0; --c)
#pragma unroll
      for (int e = S::E - 1; e >= 0; --e) arg = x[c * S::E + e] == top ? sl.index(c, e) : arg;
    arg = block_reduce<kSampleWaves>(arg, kSampleMostVocab, reinterpret_cast<int*>(buf), Least());
  } else if (top > -kInf && (binned || !ask.has_m)) {  // (with min-p alone the next kernel sums up what it leaves)
    const int cell = ask.cell(top);
    if (ask.has_k) {
#pragma unroll
      for (int e = 0; e < S::N; ++e) {
        const int b = cell - ask.cell(x[e]);
        if (b < kSampleBins - 1) atomicAdd(&bins[b], 1ull);
      }
      __syncthreads();
    } else {
      double part[NCH];
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        part[c] = 0.0;
#pragma unroll
        for (int e = 0; e < S::E; ++e) {
          const float v = x[c * S::E + e];
          const double w = ask.weight(v, top);
          part[c] += w;
          if (binned) {
            const int b = cell - ask.cell(v);
            if (b < kSampleBins - 1) atomicAdd(&bins[b], whole(w * kSliceSteps));
          }
        }
      }
      sum = sum_blocks<NCH>(part, sums, binned ? nullptr : A.blocks + at * S::kBlocks);
    }
    if (binned && tid < kSampleBins) A.hist[at * kSampleBins + tid] = ask.has_k ? (float)bins[tid] : (float)((double)bins[tid] / kSliceSteps);
  }
  if (tid == 0) A.stat[at] = SliceStat{sum, top, arg};
}

// What the slices say of a row; the lanes of one wave together.
struct RowStat {
  float top;
  double sum;  // of w, relative to the row's largest (rows without top-k)
};
__device__ __forceinline__ RowStat row_stat(const SampleArgs& A, const RowAsk& ask, int row) {
  const SliceStat* st = A.stat + (long long)row * A.nslices;
  const int lane = threadIdx.x & 63;
  RowStat r{-kInf, 0.0};
  for (int s = lane; s < A.nslices; s += 64) r.top = fmaxf(r.top, st[s].top);
  r.top = wave_reduce(r.top, -kInf, Most());
  if (!ask.greedy && !ask.has_k)
    for (int s = lane; s < A.nslices; s += 64) r.sum += st[s].sum * ask.weight(st[s].top, r.top);
  r.sum = wave_reduce(r.sum, 0.0, Add());
  return r;
}

constexpr int kSampleMostSlices = kSampleMostVocab / kSampleLargeSlice + 1;

template <typename T, int NCH>
__global__ __launch_bounds__(kSampleThreads, 8) void sample_bracket_kernel(SampleArgs A) {
  constexpr int NT = kSampleThreads;
  using S = Slice<T, NCH>;
  using L = Listed<T>;
  __shared__ double sums[2][S::kBlocks];
  constexpr int kParts = NT / kSampleBins;  // threads to a bin
  __shared__ double bins[kParts][kSampleBins], factor[kSampleMostSlices];
  __shared__ int shift[kSampleMostSlices], listed;
  const int row = blockIdx.x / A.nslices, slice = blockIdx.x - row * A.nslices, tid = threadIdx.x, lane = tid & 63;
  RowAsk ask;
  ask.init(A, row);
  if (ask.greedy || !(ask.has_k || ask.has_p || ask.has_m)) return;
  S sl;
  sl.init(A, row, slice);
  float x[S::E];
  sl.load_chunk(sl.index(0, 0), x);
  // What belongs to the row is worked out by the first wave alone: every wave at it, they would wait for each other's turn to issue
  __shared__ RowStat stat;
  __shared__ int b0_, b1_;  // tokens in bins below b0 are surely kept, those of b0 .. b1 listed
  __shared__ float sure_, list_;  // sure ones are at least `sure`, listed ones at least `list`
  const bool binned = ask.has_k || ask.has_p;
  if (tid < 64) {
    const RowStat r = row_stat(A, ask, row);
    const int cell = ask.cell(r.top);
    const SliceStat* st = A.stat + (long long)row * A.nslices;
    if (binned)
      for (int s = lane; s < A.nslices; s += 64) {
        const float top = st[s].top;
        factor[s] = top == -kInf ? 0.0 : (ask.has_k ? 1.0 : ask.weight(top, r.top));
        shift[s] = top == -kInf ? kSampleBins : cell - ask.cell(top);
      }
    if (lane == 0) {
      stat = r;
      listed = 0;
    }
  }
  __syncthreads();
  const RowStat r = stat;
  if (binned) {
    // the row's bins: two threads to each add it up over half of the slices; what lies in no bin is in the last
    const float* hist = A.hist + (long long)row * A.nslices * kSampleBins;
    static_assert(NT == 2 * kSampleBins, "half of the slices each");
    const int bin = tid & (kSampleBins - 1);
    double mine = 0.0;
#pragma unroll 4
    for (int s = tid / kSampleBins; s < A.nslices; s += kParts) {
      const int b = bin - shift[s];
      if (b >= 0 && bin < kSampleBins - 1) mine += (double)hist[s * kSampleBins + b] * factor[s];
    }
    bins[tid / kSampleBins][bin] = mine;
    __syncthreads();
  }
  if (tid < 64) {
    int b0 = kSampleBins, b1 = -1;
    if (binned) {
      // where the sum reaches what is to be kept, eight bins a lane.  Sums of w: a little less and a little more of it, for the rounding of the bins
      const double least = ask.has_k ? (double)ask.k : ask.p * r.sum * (1.0 - 1e-5), most = ask.has_k ? (double)ask.k : ask.p * r.sum * (1.0 + 1e-5);
      constexpr int PL = kSampleBins / 64;
      double v[PL], upto = 0.0;
#pragma unroll
      for (int j = 0; j < PL; ++j) {
        const int b = PL * lane + j;
        v[j] = bins[0][b] + bins[1][b];
        upto += v[j];
      }
      const double mine = upto;
      upto = wave_scan(upto, 0.0, Add()) - mine;
      int n0 = 0, n1 = 0;
#pragma unroll
      for (int j = 0; j < PL; ++j) {
        upto += v[j];
        const bool in = PL * lane + j < kSampleBins - 1;
        n0 += (int)__popcll(__ballot(in && upto < least));
        n1 += (int)__popcll(__ballot(in && upto < most));
      }
      b0 = ask.has_k ? 0 : n0;  // (what top-p takes its part of is the w of top-k's tokens: they are all listed)
      b1 = n1;
    }
    const int cell = ask.cell(r.top);
    float sure = b0 == 0 ? kInf : (b0 == kSampleBins ? -kInf : ask.edge(cell - b0 + 1));
    // min-p without top-p: of what is a little below its bound no w is wanted
    // (at very high temperatures the bound is below all finite numbers, which are then left)
    if (ask.has_m && !ask.has_p && r.top < kInf) {
      const double bound = (double)r.top + (log2(ask.f) - 1e-3) / ask.scale;
      if (bound > -3.4e38) sure = fmaxf(sure, RowAsk::next((float)bound, -1));
    }
    if (lane == 0) {
      b0_ = b0;
      b1_ = b1;
      sure_ = sure;
      list_ = b1 == kSampleBins - 1 ? -kInf : ask.edge(cell - b1);
    }
  }
  __syncthreads();
  const int b0 = b0_, b1 = b1_;
  const float sure = sure_, list = list_;
  const long long at = (long long)row * A.nslices + slice;
  typename L::Word* cand = reinterpret_cast<typename L::Word*>(A.cand) + at * S::kSize;
#pragma unroll 1
  for (int c = 0; c < NCH; ++c) {  // (one chunk at a time, the next one under way: two workgroups fit a compute unit)
    float v[S::E];
#pragma unroll
    for (int e = 0; e < S::E; ++e) v[e] = x[e];
    if (c + 1 < NCH) sl.load_chunk(sl.index(c + 1, 0), x);
    double part_all = 0.0, part = 0.0;
#pragma unroll
    for (int e = 0; e < S::E; ++e) {  // (branches that a wave takes as one)
      const bool in = v[e] > -kInf, kept = in && b0 > 0 && v[e] >= sure;
      if (__ballot(kept)) {
        const double w = kept ? ask.weight(v[e], r.top) : 0.0;
        part_all += w;
        part += w >= ask.f ? w : 0.0;
      }
      const bool open = in && !kept && b1 >= 0 && v[e] >= list;
      const u64 lanes = __ballot(open);
      if (lanes) {
        int first = 0;
        if (lane == 0) first = atomicAdd(&listed, (int)__popcll(lanes));
        first = lane_value(first, 0) + (int)__popcll(lanes & ((1ull << lane) - 1));
        if (open) cand[first] = L::pack(Rank<T>::key(v[e]), (c * NT + tid) * S::E + e);
      }
    }
    if (b0 > 0) {  // (uniform)
      part_all = wave_reduce(part_all, 0.0, Add());
      part = ask.has_m ? wave_reduce(part, 0.0, Add()) : part_all;
      if (lane == 0) {
        sums[0][c * kSampleWaves + (tid >> 6)] = part_all;
        sums[1][c * kSampleWaves + (tid >> 6)] = part;
      }
    }
  }
  __syncthreads();
  if (tid < 64) {
    const double all = b0 > 0 && lane < S::kBlocks ? sums[0][lane] : 0.0, sum = b0 > 0 && lane < S::kBlocks ? sums[1][lane] : 0.0;
    if (lane < S::kBlocks) A.blocks[at * S::kBlocks + lane] = sum;
    const double total_all = wave_reduce(all, 0.0, Add()), total = wave_reduce(sum, 0.0, Add());
    if (lane == 0) A.kept[at] = SliceKept{total_all, total, listed, 0};
  }
}

constexpr int kPickBins = 256;     // of a round of the selection
constexpr int kPickList = 7680;    // listed tokens that stay in LDS; longer lists are looked up again for every pass (4 rows of 7680 equal logits 72 us, of 9000 102)

struct PickLds {
  u64 buf[kSampleWaves];
  u64 bins[2][kPickBins];        // in use, and cleared meanwhile: these four
  uint32_t least_key[2], most_key[2];
  int few[2];
  ulonglong2 few_of[64];           // (rank, amount)
  u64 above[64];                   // amount, number of the others above each of them: zero but while in use
  int place[64];
  u64 lo, hi, before, result;
  u64 rank[kPickList];
  u64 steps[kPickList];            // w in steps
  uint16_t slice[kPickList];
  int first[kSampleMostSlices + 1];  // the slices' first places in the list
  u64 kept[kSampleMostSlices];     // steps of the listed tokens that are left
  u64 block[64];                   // the same of the blocks of the chosen slice
  u64 total;
  double sums[kSampleMostSlices];  // w of the slices that is left
};

template <typename T, int NCH>
__global__ __launch_bounds__(kSampleThreads) void sample_pick_kernel(SampleArgs A, int filtered) {
  constexpr int NT = kSampleThreads;
  using S = Slice<T, NCH>;
  using L = Listed<T>;
  __shared__ PickLds lds;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  RowAsk ask;
  ask.init(A, row);
  const long long at = (long long)row * A.nslices;
  const bool cuts = filtered && !ask.greedy && (ask.has_k || ask.has_p), sums = filtered && (cuts || ask.has_m);
  int listed = 0;
  if (cuts) {  // how many each slice has listed, and what they have surely kept
    for (int s = tid; s < A.nslices; s += NT) {
      lds.first[s + 1] = A.kept[at + s].listed;
      lds.sums[s] = A.kept[at + s].all;
      lds.kept[s] = 0;
    }
    if (tid < 64) {
      lds.block[tid] = 0;
      lds.above[tid] = 0;
      lds.place[tid] = 0;
    }
    if (tid < 2) {
      lds.least_key[tid] = ~0u;
      lds.most_key[tid] = 0;
      lds.few[tid] = 0;
    }
    for (int b = tid; b < 2 * kPickBins; b += NT) (&lds.bins[0][0])[b] = 0;
    if (tid == 0) lds.first[0] = 0, lds.total = 0;
  }
  __shared__ RowStat stat;
  if (tid < 64) {  // (see the kernel before)
    const RowStat r = row_stat(A, ask, row);
    if (lane == 0) stat = r;
  }
  __syncthreads();
  const RowStat r = stat;
  if (r.top == -kInf) {
    if (tid == 0) {
      A.token[row] = -1;
      if (A.logprob) A.logprob[row] = -kInf;
    }
    return;
  }
  if (ask.greedy) {
    int arg = kSampleMostVocab;
    for (int s = lane; s < A.nslices; s += 64)
      if (A.stat[at + s].top == r.top) arg = min(arg, A.stat[at + s].arg);
    arg = wave_reduce(arg, kSampleMostVocab, Least());
    if (tid == 0) {
      A.token[row] = arg;
      if (A.logprob) A.logprob[row] = 0.f;
    }
    return;
  }
  u64 cut = 0;  // tokens of this rank and above are left by top-k and top-p
  double steps = 1.0;  // steps of w that make 1
  if (cuts) {
    if (tid < 64) {  // sums up to and with each slice
      int run = 0;
      for (int s0 = 0; s0 < A.nslices; s0 += 64) {
        const int s = s0 + lane;
        const int n = wave_scan(s < A.nslices ? lds.first[s + 1] : 0, 0, Add());
        if (s < A.nslices) lds.first[s + 1] = run + n;
        run += lane_value(n, 63);
      }
    }
    __syncthreads();
    listed = lds.first[A.nslices];
    steps = exp2((double)(62 - (32 - __clz(listed | 1))));  // (w <= 1: sums stay below 2^63)
  }
  const bool held = listed <= kPickList;
  const int from0 = -(int)((reinterpret_cast<uintptr_t>(reinterpret_cast<const T*>(A.logits) + (long long)row * A.stride) & 15u) / sizeof(T));
  // (rounded up: a token with any w can be drawn, by a random number of 0 if by no other)
  auto in_steps = [&](float x) { return (u64)ceil(ask.weight(x, r.top) * steps); };
  // every listed token: fn(rank, w in steps, slice)
  auto each = [&](auto fn) {
    if (held) {
      for (int i = tid; i < listed; i += NT) fn(lds.rank[i], lds.steps[i], (int)lds.slice[i]);
      return;
    }
    for (int s = 0; s < A.nslices; ++s) {
      const int n = lds.first[s + 1] - lds.first[s];
      const typename L::Word* cand = reinterpret_cast<const typename L::Word*>(A.cand) + (at + s) * S::kSize;
#pragma unroll 4
      for (int i = tid; i < n; i += NT) {
        const typename L::Word w = cand[i];
        fn(Rank<T>::of(L::key(w), from0 + s * S::kSize + L::place(w)), in_steps(Rank<T>::logit(L::key(w))), s);
      }
    }
  };
  int turn = 0;  // which of the two sets of bins and limits is in use
  // Of the listed tokens of rank >= least and with an amount: the rank of the last one in falling order before which the amounts add up to less than
  // `target` (at least 1).  Bins over the ranks narrow them down to at most 64, which are compared with each other.
  auto select = [&](u64 target, u64 least, auto amount) {
    u64 before = 0;  // amount of the ranks above those that are left
    bool few = listed <= 64;
    int n = listed;
    if (!few) {
      uint32_t least_key = ~0u, most_key = 0;
      each([&](u64 k, u64 w, int) {
        if (k < least || amount(w) == 0) return;
        const uint32_t key = (uint32_t)(k >> 22);
        least_key = min(least_key, key);
        most_key = max(most_key, key);
      });
      least_key = wave_reduce(least_key, ~0u, Least());
      most_key = wave_reduce(most_key, 0u, Most());
      if (lane == 0) {
        atomicMin(&lds.least_key[turn], least_key);
        atomicMax(&lds.most_key[turn], most_key);
      }
      __syncthreads();
      least_key = lds.least_key[turn];
      most_key = lds.most_key[turn];
      if (least_key > most_key) return least;  // (none has an amount; nothing was changed)
      u64 lo = (u64)least_key << 22, hi = ((u64)most_key << 22) | (kSampleMostVocab - 1);
      while (!few) {  // the rank is in lo .. hi, which agree above bit `shift + 8`
        const int shift = max(0, 64 - __clzll((long long)(lo ^ hi)) - 8);
        each([&](u64 k, u64 w, int) {
          if (k >= lo && k <= hi && k >= least) atomicAdd(&lds.bins[turn][(k >> shift) & 255], amount(w));
        });
        if (tid < kPickBins) lds.bins[turn ^ 1][tid] = 0;
        if (tid == 0) {
          lds.least_key[turn ^ 1] = ~0u;
          lds.most_key[turn ^ 1] = 0;
        }
        __syncthreads();
        // (every wave reads it behind the last barrier of a round: cleared sooner, a late one would see none and leave the loop alone)
        if (tid == 0) lds.few[turn ^ 1] = 0;
        // bins from the highest down: the last one with something in it, before which the sum is below the target
        if (tid < 64) {
          u64 v[4], mine = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j] = lds.bins[turn][255 - 4 * lane - j];
            mine += v[j];
          }
          u64 sum = before + wave_scan(mine, (u64)0, Add()) - mine, b_before = 0;
          int b = -1;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (v[j] != 0 && sum < target) {
              b = 255 - 4 * lane - j;
              b_before = sum;
            }
            sum += v[j];
          }
          const int last = 63 - __clzll((long long)__ballot(b >= 0));
          if (lane == last) {
            const u64 base = ((lo >> shift) & ~255ull) + (u64)b;
            lds.before = b_before;
            lds.lo = max(lo, base << shift);
            lds.hi = min(hi, ((base + 1) << shift) - 1);
          }
        }
        __syncthreads();
        before = lds.before;
        lo = lds.lo;
        hi = lds.hi;
        each([&](u64 k, u64 w, int) {
          if (k < lo || k > hi || k < least || amount(w) == 0) return;
          const int at = atomicAdd(&lds.few[turn], 1);
          if (at < 64) lds.few_of[at] = make_ulonglong2(k, amount(w));
        });
        __syncthreads();
        n = lds.few[turn];
        few = n <= 64;
        turn ^= 1;
      }
    }
    auto of = [&](int i) {
      if (listed > 64) return lds.few_of[i];
      return make_ulonglong2(lds.rank[i], lds.rank[i] < least ? 0 : amount(lds.steps[i]));
    };
    const ulonglong2 mine = lane < n ? of(lane) : make_ulonglong2(0, 0);
    u64 above = 0;
    int place = 0;
    for (int j = tid >> 6; j < n; j += kSampleWaves) {
      const ulonglong2 x = of(j);
      above += x.x > mine.x ? x.y : 0;
      place += x.x > mine.x && x.y != 0 ? 1 : 0;
    }
    if (lane < n) {
      atomicAdd(&lds.above[lane], above);
      atomicAdd(&lds.place[lane], place);
    }
    __syncthreads();
    if (tid < 64) {
      above = before + lds.above[lane];
      place = lds.place[lane];
      lds.above[lane] = 0;
      lds.place[lane] = 0;
      const u64 kept = __ballot(mine.y != 0 && above < target);  // the first ones in falling order
      const bool end = mine.y != 0 && place == (int)__popcll(kept) - 1;
      if (kept == 0 ? lane == 0 : end) lds.result = kept == 0 ? least : mine.x;
    }
    __syncthreads();
    return lds.result;
  };
  // steps of a listed token that top-k, top-p and min-p leave
  auto left_of = [&](u64 k, u64 w) -> u64 {
    if (k < cut) return 0;
    return !ask.has_m || ask.weight(Rank<T>::logit((uint32_t)(k >> 22)), r.top) >= ask.f ? w : 0;
  };
  if (cuts) {
    if (held) {
      for (int i = tid; i < listed; i += NT) {
        int lo = 0, n = A.nslices;  // the last slice with first <= i
        while (n > 1) {
          const int half = n >> 1;
          const bool up = lds.first[lo + half] <= i;
          lo += up ? half : 0;
          n = up ? n - half : half;
        }
        const typename L::Word w = reinterpret_cast<const typename L::Word*>(A.cand)[(at + lo) * S::kSize + (i - lds.first[lo])];
        lds.rank[i] = Rank<T>::of(L::key(w), from0 + lo * S::kSize + L::place(w));
        lds.steps[i] = in_steps(Rank<T>::logit(L::key(w)));
        lds.slice[i] = (uint16_t)lo;
      }
      __syncthreads();
    }
    if (ask.has_k && listed >= ask.k) cut = select((u64)ask.k, 0, [](u64) { return 1ull; });
    if (ask.has_p) {
      double total = r.sum, before = 0.0;  // of what top-k leaves, and of what is surely kept
      if (ask.has_k) {
        u64 t = 0;
        each([&](u64 k, u64 w, int) { t += k >= cut ? w : 0; });
        t = wave_reduce(t, (u64)0, Add());
        if (lane == 0) atomicAdd(&lds.total, t);
        __syncthreads();
        total = (double)lds.total / steps;
      } else {
        for (int s = lane; s < A.nslices; s += 64) before += lds.sums[s];
        before = wave_reduce(before, 0.0, Add());
      }
      // (whole steps before a token are fewer than the target's if they are fewer than it rounded up; the first token stays.  Sums that are equal, as among
      // equal logits, must not be told apart by their rounding: a little less than the target)
      const double target = ceil((ask.p * total * (1.0 - kRounding) - before) * steps);
      if (listed > 0) cut = max(cut, select(target >= 1.0 ? (u64)target : 1ull, cut, [](u64 w) { return w; }));
    }
    if (held) {  // (a slice's tokens follow one another: a wave sums them up)
      for (int s = tid >> 6; s < A.nslices; s += kSampleWaves) {
        u64 t = 0;
        for (int i = lds.first[s] + lane; i < lds.first[s + 1]; i += 64) t += left_of(lds.rank[i], lds.steps[i]);
        t = wave_reduce(t, (u64)0, Add());
        if (lane == 0) lds.kept[s] = t;
      }
    } else {
      each([&](u64 k, u64 w, int s) {
        const u64 t = left_of(k, w);
        if (t) atomicAdd(&lds.kept[s], t);
      });
    }
    __syncthreads();
  }
  // ---------------------------------------------------------------- the slice that the random number falls into (the first wave)
  __shared__ int chosen;
  __shared__ double left;  // of the random number's share in the chosen slice
  __shared__ double all;
  if (tid < 64) {
    const float un = A.uniform[row];
    const double u = (opaque_bits(un) & 0x7fffffffu) > 0x7f800000u ? 0.0 : fmin(fmax((double)un, 0.0), 1.0);
    double total = 0.0;
    for (int s0 = 0; s0 < A.nslices; s0 += 64) {
      const int s = s0 + lane;
      double x = 0.0;
      if (s < A.nslices) {
        x = sums ? A.kept[at + s].sum : A.stat[at + s].sum * ask.weight(A.stat[at + s].top, r.top);
        if (cuts) x += (double)lds.kept[s] / steps;
        lds.sums[s] = x;
      }
      total += wave_reduce(x, 0.0, Add());
    }
    const double want = u * total * (1.0 + kRounding);
    double run = 0.0, rest = 0.0;
    int pick = -1;
    bool done = false;
    for (int s0 = 0; s0 < A.nslices && !done; s0 += 64) {  // the first slice up to and with which the sum is more; else the last with something in it
      const int s = s0 + lane;
      const double x = s < A.nslices ? lds.sums[s] : 0.0;
      const double upto = wave_scan(x, 0.0, Add());
      const double before = run + (upto - x);
      const u64 over = __ballot(x > 0.0 && run + upto > want), some = __ballot(x > 0.0);
      const int l = over ? __builtin_ctzll(over) : 63 - __clzll((long long)some);
      if (over || some) {
        pick = s0 + l;
        rest = want - lane_value(before, l);
      }
      done = over != 0;
      run += lane_value(upto, 63);
    }
    if (lane == 0) {
      chosen = pick;
      left = rest;
      all = total;
    }
  }
  __syncthreads();
  // ---------------------------------------------------------------- the block in it, and the token
  if (cuts && held) {
    for (int i = lds.first[chosen] + tid; i < lds.first[chosen + 1]; i += NT) {
      const u64 t = left_of(lds.rank[i], lds.steps[i]);
      const int index = kSampleMostVocab - 1 - (int)(lds.rank[i] & (kSampleMostVocab - 1));
      if (t) atomicAdd(&lds.block[(index - from0 - chosen * S::kSize) / S::kBlock], t);
    }
  } else if (cuts) {
    const typename L::Word* cand = reinterpret_cast<const typename L::Word*>(A.cand) + (at + chosen) * S::kSize;
    for (int i = tid; i < lds.first[chosen + 1] - lds.first[chosen]; i += NT) {
      const float x = Rank<T>::logit(L::key(cand[i]));
      const u64 t = left_of(Rank<T>::of(L::key(cand[i]), from0 + chosen * S::kSize + L::place(cand[i])), in_steps(x));
      if (t) atomicAdd(&lds.block[L::place(cand[i]) / S::kBlock], t);
    }
  }
  if (cuts) __syncthreads();
  if (tid >= 64) return;
  const double want = left;
  double x = 0.0;
  if (lane < S::kBlocks) {
    x = A.blocks[(at + chosen) * S::kBlocks + lane] * (sums ? 1.0 : ask.weight(A.stat[at + chosen].top, r.top));
    if (cuts) x += (double)lds.block[lane] / steps;
  }
  {
    const double upto = wave_scan(x, 0.0, Add());
    const u64 over = __ballot(x > 0.0 && upto > want);
    u64 some = __ballot(x > 0.0), past, any;
    int l = over ? __builtin_ctzll(over) : 63 - __clzll((long long)some);  // (else the sum of the blocks fell just short of the slice's)
    S sl;
    sl.init(A, row, chosen);
    int i0;
    float v[S::E];
    double w[S::E], sum, to, rest;
    for (;;) {
      rest = want - lane_value(upto - x, l);
      i0 = from0 + chosen * S::kSize + l * S::kBlock + lane * S::E;
      sl.load_chunk(i0, v);
      sum = 0.0;
#pragma unroll
      for (int e = 0; e < S::E; ++e) {
        w[e] = ask.weight(v[e], r.top);
        if (!(w[e] >= ask.f) || Rank<T>::of(v[e], i0 + e) < cut) w[e] = 0.0;
        sum += w[e];
      }
      to = wave_scan(sum, 0.0, Add());
      past = __ballot(sum > 0.0 && to > rest);
      any = __ballot(sum > 0.0);
      // A block's sum next to the slice's largest may be a number where w next to the row's largest is less than 2^-1074 for each of its tokens: the next block,
      // or else the one before.  (The block with the slice's largest has a token; the random number is 0 or 1 where this counts.)
      some &= ~(1ull << l);
      if (any || some == 0) break;
      const u64 behind = some & (~0ull << l);
      l = behind ? __builtin_ctzll(behind) : 63 - __clzll((long long)some);
    }
    const int mine = past ? __builtin_ctzll(past) : 63 - __clzll((long long)any);
    if (lane == mine) {
      double t = to - sum, drawn = 0.0;
      int token = -1;
      bool done = false;
#pragma unroll
      for (int e = 0; e < S::E; ++e) {
        t += w[e];
        if (w[e] > 0.0 && !done) {
          token = i0 + e;
          drawn = w[e];
          done = t > rest;
        }
      }
      A.token[row] = token;
      if (A.logprob) A.logprob[row] = (float)log(drawn / all);
    }
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
  // (rows that begin at round addresses need no room for slices that do not)
  const bool round = (reinterpret_cast<uintptr_t>(logits) & 15u) == 0 && (p->rows == 1 || p->stride * (int64_t)es % 16 == 0);
  a.nslices = round ? ceil_div(p->vocab, L.slice) : L.nslices;
  a.stride = p->stride;
  a.stat = reinterpret_cast<SliceStat*>(ws + L.off_stat);
  a.hist = reinterpret_cast<float*>(ws + L.off_hist);
  a.kept = reinterpret_cast<SliceKept*>(ws + L.off_kept);
  a.blocks = reinterpret_cast<double*>(ws + L.off_blocks);
  a.cand = ws + L.off_cand;
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
