// Softmax attention of new tokens over a paged cache: o_i = sum_j p_ij v_j, p_ij = exp(s_ij - lse_i), with the scales, bias and masks of the entmax
// attention and, if asked for, scores capped by a tanh.  One pass over keys and values: a row's largest score and sum so far, its output so far
// scaled down whenever a much larger score comes.  Scores as in the tiled kernel there, S^T = K Q^T with a lane pair for each of 32 folded rows (token, head of the
// group), whose probabilities are the second operand of O^T = V^T P^T as they are.
//   softmax_split_piece()  sequences of at most kSplitRows folded rows (decode steps): the keys are cut into pieces, a workgroup each.  A wave
//                          goes through 32-key tiles of its own, brought to LDS by loads that it alone waits for; the waves meet at the end.
//                          Bound by the one read of K and V: 48 sequences of 150 to 9000 keys, 2 heads of 128, 23 us (4.1 TB/s); two of 65536 keys, 4 heads, 50 us (5.4 TB/s).
//   softmax_tiled_piece()  others: a workgroup per 128 folded rows and piece of the keys, tiles of keys and values shared by its waves; bound by the matrix
//                          products, of which the one with V is made twice in bf16
//   softmax_join_kernel    adds up the pieces' outputs, each in units of its own reference score
// Both kinds of pieces have a kernel of their own and one for calls that have both.
#pragma once
#include "launch.hip.h"
#include "seq.hip.h"
#include "seq_tiled.hip.h"
#include "softmax_layout.h"

namespace entmax {

struct SoftmaxCall {
  const entmax_seq_params* p;
  float cap;
  const void *Q, *K, *V;
  const int32_t *cu, *kv_len, *table;
  const float *beta, *gamma, *slopes;
  void* O;
  float* lse;
  char* ws;
  hipStream_t st;
};

struct SoftmaxArgs {
  SeqGeom g;  // (alpha 2: y = s)
  const void *Q, *K, *V;
  void* O;
  float* lse;
  float cap;
  float* part;    // [places][rows][D], a place for every piece: see SoftmaxShare
  float2* sums;   // [places][rows] (largest score in units of log 2, sum)
  int2* shares;   // (shared) [nseq] first and n of the sequences' SoftmaxShare
  int rows;
  int shared;     // pieces from the lengths of all sequences (else of `piece` keys, `splits` to a sequence)
  int budget, least;  // shared: tiles are dealt out to about so many workgroups, at least so many to each
  int piece, splits;
  int nblk;
  int split;      // sequences with few rows are left to softmax_split_kernel
  float* tpart;   // softmax_tiled_kernel: [nblk][Hkv][tsplits][128][D], [..][128], as part and sums
  float2* tsums;
  int tpiece, tsplits;  // keys of a workgroup (a multiple of 64) and the most pieces of a group
};

// How a sequence's keys are cut up: n equal pieces of `len` keys, whole tiles of 32 (one piece of none if there are no keys).  Piece k of key/value head hk has place
// (first + k) Hkv + hk.
struct SoftmaxShare {
  int first, n, len;
  __device__ __forceinline__ void cut(int keys, int most_tiles, int step = 1) {  // (pieces of whole steps of tiles)
    const int tiles = (keys + 31) >> 5;
    n = max(1, (tiles + most_tiles - 1) / most_tiles);
    const int each = ((tiles + n - 1) / n + step - 1) / step * step;
    if (each > 0) n = max(1, (tiles + each - 1) / each);
    len = each * 32;
  }
};

// The share of the sequence that has place x, with what it is; false: there is none.
// Memory delivers as much as it can when all compute units ask for equal parts of it at the same time, and the host knows only a bound of the lengths: so
// every wave adds up the tiles of all sequences (64 at a time, a lane each), divides them by the number of workgroups that fit the chip, and
// numbers the pieces that come of it.  (48 sequences of 150 to 9000 keys, 2 heads of 128: 41 us with pieces by the bound, 31 so.)  With many
// sequences that would take longer than it gives: pieces by the bound.
__device__ __forceinline__ bool softmax_share(const SoftmaxArgs& A, int x, SeqView& v, SoftmaxShare& sh) {
  const SeqGeom& g = A.g;
  if (!A.shared) {
    const int s = x / A.splits;
    if (s >= g.nseq || !load_seq(g, s, v) || !split_seq(g, v)) return false;
    sh.cut(v.L, A.piece >> 5);
    sh.first = s * A.splits;
    return true;
  }
  const int lane = threadIdx.x & 63;
  auto load = [&](int s, SeqView& t) {
    const bool ok = s < g.nseq && load_seq(g, s, t) && split_seq(g, t);
    return ok ? max(1, (t.L + 31) >> 5) : 0;
  };
  SeqView t;
  int tiles = load(lane, t);
  long long all = tiles;
  for (int s0 = 64; s0 < g.nseq; s0 += 64) {
    SeqView u;
    all += load(s0 + lane, u);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) all += __shfl_xor(all, off);
  const int most = max(A.least, (int)((all * g.Hkv + A.budget - 1) / A.budget));
  int first = 0;
  for (int s0 = 0; s0 < g.nseq; s0 += 64) {
    if (s0) tiles = load(s0 + lane, t);
    SoftmaxShare mine;
    mine.cut(t.L, most);
    if (tiles == 0) mine.n = 0;
    int upto = mine.n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(upto, off);
      if (lane >= off) upto += y;
    }
    const unsigned long long here = __ballot(first + upto > x);
    if (here) {
      const int l = __builtin_ctzll(here);
      v.s = s0 + l;
      v.row0 = __builtin_amdgcn_readlane(t.row0, l);
      v.n = __builtin_amdgcn_readlane(t.n, l);
      v.L = __builtin_amdgcn_readlane(t.L, l);
      sh.n = __builtin_amdgcn_readlane(mine.n, l);
      sh.len = __builtin_amdgcn_readlane(mine.len, l);
      sh.first = first + __builtin_amdgcn_readlane(upto, l) - sh.n;
      return sh.n > 0;
    }
    first += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A cap above this is none: c tanh(s / c) is s to a step of a float up to c / 4096, 2^52, and exponentials of numbers of that size are 0 or 1 either way.  (From
// 2e38 on the cap itself would leave the range of a float in units of log 2, and s / c that of whole ones.)
constexpr float kSoftmaxMostCap = 18446744073709551616.f;
// bf16: up to this cap 1.2e-7 of it is no more than the 2^-17 or so that probabilities as two bf16 numbers are off by, and tanh needs no series near zero.  (4 x 700 tokens against
// 6000 keys, 4 x 4 heads of 128, cap 30: 333 us, 387 with the series.)
constexpr float kSoftmaxPlainCap = 64.f;

// From accumulators of the dot products to scores in units of log 2: score = unit * x, x the accumulator or, with a cap, what capped() makes of it.
template <typename T, bool CAP>
struct SoftmaxScale {
  float unit, slack;      // slack: x of a factor of 2^24
  float cap2, in2, late;  // CAP: cap in units of log 2; s / cap = in2 * accumulator; slope of a bias outside the cap
  bool series;            // CAP: the same in all lanes
  // a, w: as in SeqRow; w is zero afterwards if the bias is added late
  __device__ __forceinline__ void init_scale(const SoftmaxArgs& A, float a, float& w) {
    unit = CAP ? 1.f : a * kLog2e;
    slack = fminf(24.f / unit, 1e30f);
    if (CAP) {
      cap2 = A.cap * kLog2e;
      in2 = fminf(a / A.cap, 3e38f);  // (no infinity that a product of 0 would meet)
      late = 0.f;
      series = A.cap > kSoftmaxPlainCap;
      if (A.g.bias_mode == 1) {
        late = a * w * kLog2e;
        w = 0.f;
      }
    }
  }
  // SERIES: see kSoftmaxPlainCap
  template <bool SERIES>
  __device__ __forceinline__ float capped(float acc, int dist) const {
    // 1 - 2 / (1 + exp(2 x)): off by some 1.2e-7, of the cap.  SERIES: near zero, where that is much of the value (all of it with a cap far above the scores), the
    // first five terms of the series (the sixth is 1e-8 of it at 1/4)
    const float x = acc * in2;
    float t = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * kLog2e)));
    if constexpr (SERIES) {
      const float x2 = x * x;
      const float near = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
      t = x2 < 0.0625f ? near : t;
    }
    return fmaf(late, (float)max(dist, 0), cap2 * t);
  }
  // N scores, dist(e) the distance of the e-th
  template <int N, typename V, class F>
  __device__ __forceinline__ void cap_all(V& x, F dist) const {
    if (sizeof(T) == 4 || series) {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = capped<true>(x[e], dist(e));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = capped<false>(x[e], dist(e));
    }
  }
};

// An address that is the same in all lanes, as one
__device__ __forceinline__ const char* uniform(const char* at) {
  const unsigned long long x = (unsigned long long)at;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (const char*)((unsigned long long)hi << 32 | lo);
}

// Eight numbers as sums of two bf16 ones each, in pairs
__device__ __forceinline__ void split_pairs(const float* x, Frag<bf16_t>& hi, Frag<bf16_t>& lo) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x[2 * e], x[2 * e + 1]}), bf16x2_t));
    const f32x2_t rest = {x[2 * e] - __uint_as_float(h << 16), x[2 * e + 1] - __uint_as_float(h & 0xffff0000u)};
    hi.v[e] = h;
    lo.v[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2_t));
  }
}

// The larger of x in this lane and in the one 32 lanes away
__device__ __forceinline__ float other_half_max(float x) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// A wave's 32 rows, a lane pair each, and what they have seen so far.
template <typename T, int D, bool CAP>
struct SoftmaxRows : SeqRows<T, D>, SoftmaxScale<T, CAP> {
  static constexpr int kRows = 32, NC = D / 16, NM = D / 32;
  static constexpr int kChunks = NM * 4;  // a lane's parts of the output, four features each
  static constexpr int kProbs = 16;       // a lane's probabilities of 32 keys
  float top, sum;    // x that none of the scores so far is above; sum of this lane's exp2(unit (x - top))
  f32x16_t oacc[NM];
  __device__ __forceinline__ void init(const SoftmaxArgs& A, const SeqView& v, int hk, int r0) {
    SeqRows<T, D>::init(A.g, v, A.Q, hk, r0);
    this->init_scale(A, this->a, this->w);
    this->biased = __ballot(this->w != 0.f) != 0ull;
    top = -kInf;
    sum = 0.f;
#pragma unroll
    for (int mm = 0; mm < NM; ++mm)
      oacc[mm] = f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ int row() const { return this->li; }
  __device__ __forceinline__ bool first_lane() const { return this->hh == 0; }
  __device__ __forceinline__ float total() const { return sum + __shfl_xor(sum, 32); }
  __device__ __forceinline__ int feature(int chunk) const { return 8 * chunk + 4 * this->hh; }
  __device__ __forceinline__ f32x4_t out(int chunk) const {
    const f32x16_t& o = oacc[chunk >> 2];
    const int e = 4 * (chunk & 3);
    return f32x4_t{o[e], o[e + 1], o[e + 2], o[e + 3]};
  }
  // S^T of 32 keys as in SeqRows; fp32: sums of sixteen features each, one after the other so that few of them are held, added up as a tree
  template <class F>
  __device__ __forceinline__ f32x16_t scores(f32x16_t acc, F frag) const {
    if constexpr (sizeof(T) == 2) return this->dots(acc, frag);
    else return acc + branch<0, NC>(frag);
  }
  template <int FROM, int N, class F>
  __device__ __forceinline__ f32x16_t branch(F frag) const {
    if constexpr (N > 1) {
      const f32x16_t left = branch<FROM, N / 2>(frag);
      __builtin_amdgcn_sched_barrier(0);
      const f32x16_t right = branch<FROM + N / 2, N / 2>(frag);
      return left + right;
    } else {
      return Elem<T>::mma(frag(FROM), this->qf[FROM], f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f});
    }
  }
  __device__ __forceinline__ void cap_scores(f32x16_t& acc, int j0) const {
    this->template cap_all<16>(acc, [&](int e) { return this->pos - j0 - this->key_of(e); });
  }
  __device__ __forceinline__ void add_bias(f32x16_t& acc, int j0) const {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = fmaf(this->w, (float)max(this->pos - j0 - this->key_of(e), 0), acc[e]);
  }
  // Moves `top` to 2^24 times the largest score if some score x = acc (masked ones -inf) is above it.  No probability is above 1 then, so that the sums overflow
  // no sooner than those of exp(s - max) v would; the largest is 2^-24 at least, so that none that counts is lost at 2^-126; and the sums are rarely scaled anew.  It
  // costs accuracy: exponents near -24 are rounded to 2^-20, probabilities to 6.6e-7 of them instead of 6e-8.
  template <int NB>
  __device__ __forceinline__ void raise(const f32x16_t (&acc)[NB]) {
    const float m = other_half_max(most(acc));
    const bool more = m > top;
    if (__ballot(more) != 0ull) {
      const float to = m + this->slack, f = more ? __builtin_amdgcn_exp2f((top - to) * this->unit) : 1.f;  // (0 from -inf)
      top = more ? to : top;
      sum *= f;
#pragma unroll
      for (int mm = 0; mm < NM; ++mm)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[mm][e] *= f;
    }
  }
  // whether raise() would
  template <int NB>
  __device__ __forceinline__ bool rises(const f32x16_t (&acc)[NB]) const {
    return __ballot(most(acc) > top) != 0ull;
  }
  template <int NB>
  static __device__ __forceinline__ float most(const f32x16_t (&acc)[NB]) {
    float m = max16(acc[0]);
#pragma unroll
    for (int b = 1; b < NB; ++b) m = fmaxf(m, max16(acc[b]));
    return m;
  }
  // p = exp2(score - top) of eight of a block's scores, added to the sum
  __device__ __forceinline__ void probs8(const f32x16_t& acc, int from, float* p) {
    const float base = top > -kInf ? -top * this->unit : 0.f;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(acc[from + e], this->unit, base));
      p[e + 1] = __builtin_amdgcn_exp2f(fmaf(acc[from + e + 1], this->unit, base));
      s0 += p[e];
      s1 += p[e + 1];
    }
    sum += s0 + s1;
  }
  __device__ __forceinline__ void probs(const f32x16_t& acc, float (&p)[16]) {
    probs8(acc, 0, p);
    probs8(acc, 8, p + 8);
  }
  __device__ __forceinline__ float top2() const { return top > -kInf ? top * this->unit : -kInf; }

  // ---- the 32 keys and values of a wave's own tile
  using KTile = SeqTile<T, D, 32, false, 64>;
  using Vals = SeqValues<T, D, 32, 64>;
  using VTile = typename Vals::VT;
  struct Places {
    FragOff<T> k[NC];
    Vals v;
    __device__ __forceinline__ void init(int lane) {
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) k[cc] = FragOff<T>::template make<typename KTile::Tile>(lane & 31, 2 * cc + (lane >> 5));
      v.init(lane);
    }
  };
  // whether some row does not see some key
  __device__ __forceinline__ bool take_keys(const Places& at, const char* tile, int j0, const SeqKeys& keys, bool hole, float (&p)[kProbs]) {
    f32x16_t acc[1] = {scores(this->start(j0), [&](int cc) { return at.k[cc].load(tile, 0); })};
    if constexpr (CAP) cap_scores(acc[0], j0);
    const bool masked = hole || j0 + 32 > this->lim_min;
    if (masked) this->mask(acc[0], j0, keys, hole);
    raise<1>(acc);
    probs(acc[0], p);
    return masked;
  }
  __device__ __forceinline__ void take_values(const Places& at, const char* tile, const float (&p)[kProbs], bool masked) {
    at.v.accumulate(tile, 0, p, masked, oacc);
  }
};

// A wave's 16 rows, four lanes each, on the matrix instructions of 16 x 16: half the work of SoftmaxRows where there are not more rows.  (48 sequences of 150 to
// 9000 keys: 31 us, 33 with 32 rows; 256 to 2000 keys: 66 and 77; 12 of three tokens in fp32, capped: 29 and 53.)
// Lane l has row l % 16; of 32 keys those of 16 (e / 4) + 4 (l / 16) + e % 4, e = 0 .. 7, and of the output features 16 f + 4 (l / 16) + 0 .. 3.
template <typename T, int D, bool CAP>
struct SoftmaxRows16 : SeqRow, SoftmaxScale<T, CAP> {
  static constexpr int kRows = 16, kChunks = D / 16, kProbs = 8;
  static constexpr int NC = D * (int)sizeof(T) / 64;  // fragments of a row of queries or keys, 16 bytes of a lane
  using KTile = SeqTile<T, D, 32, false, 64>;
  using VTile = SeqTile<T, D, 32, sizeof(T) == 2, 64>;
  int lane, li, quad, lim_min, lim_max;
  bool biased;
  u32x4_t qf[NC];
  float top, sum;
  f32x4_t oacc[kChunks];
  __device__ __forceinline__ void init(const SoftmaxArgs& A, const SeqView& v, int hk, int r0) {
    lane = threadIdx.x & 63;
    li = lane & 15;
    quad = lane >> 4;
    SeqRow::init<sizeof(T) == 2>(A.g, v, hk, r0 + li, D);
    this->init_scale(A, a, w);
    biased = __ballot(w != 0.f) != 0ull;
    lim_min = __builtin_amdgcn_readfirstlane(lim);  // (limits do not decrease from row to row)
    const int last = min(v.n * A.g.G - 1 - r0, 15);
    lim_max = last < 0 ? 0 : __builtin_amdgcn_readlane(lim, last);
    const char* q = reinterpret_cast<const char*>(reinterpret_cast<const T*>(A.Q) + (long long)(v.row0 + t) * A.g.q_st + (long long)head * A.g.q_sh);
    const uint32_t sign = c < 0.f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) {
      qf[cc] = *reinterpret_cast<const u32x4_t*>(q + 64 * cc + 16 * quad);
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[cc][e] = c != 0.f ? qf[cc][e] ^ sign : 0u;  // (0 beyond the last row, too)
    }
    top = -kInf;
    sum = 0.f;
#pragma unroll
    for (int f = 0; f < kChunks; ++f) oacc[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ int row() const { return li; }
  __device__ __forceinline__ bool first_lane() const { return quad == 0; }
  __device__ __forceinline__ float total() const {
    const float x = sum + __shfl_xor(sum, 16);
    return x + __shfl_xor(x, 32);
  }
  __device__ __forceinline__ int feature(int chunk) const { return 16 * chunk + 4 * quad; }
  __device__ __forceinline__ f32x4_t out(int chunk) const { return oacc[chunk]; }
  __device__ __forceinline__ float top2() const { return top > -kInf ? top * this->unit : -kInf; }
  __device__ __forceinline__ int key_of(int e) const { return 16 * (e >> 2) + 4 * quad + (e & 3); }
  struct Places {
    int k[NC], v[sizeof(T) == 2 ? kChunks : 1];
    __device__ __forceinline__ void init(int lane) {
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) k[cc] = KTile::off(lane & 15, 4 * cc + (lane >> 4));
      if constexpr (sizeof(T) == 2) {  // (see SeqValues)
        const int p = lane & 15, row = 4 * (lane >> 4) + (p >> 2);
#pragma unroll
        for (int f = 0; f < kChunks; ++f) v[f] = VTile::off(row, 2 * f + ((p & 3) >> 1)) + (p & 1) * 8;
      }
    }
  };
  template <int FROM, int N>
  static __device__ __forceinline__ f32x4_t branch(const f32x4_t* x) {
    if constexpr (N > 1) return branch<FROM, N / 2>(x) + branch<FROM + N / 2, N / 2>(x);
    else return x[FROM];
  }
  // S^T of keys 16 b .. 16 b + 15 of the tile, on top of acc
  __device__ __forceinline__ f32x4_t scores(const Places& at, const char* tile, int b, f32x4_t acc) const {
    const char* from = tile + 16 * b * KTile::kRowBytes;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int cc = 0; cc < NC; ++cc)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(from + at.k[cc])),
                                                      __builtin_bit_cast(bf16x8_t, qf[cc]), acc, 0, 0, 0);
      return acc;
    } else {  // (sums of sixteen features each, added up as a tree: see SoftmaxRows)
      f32x4_t part[NC];
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) {
        const f32x4_t k = *reinterpret_cast<const f32x4_t*>(from + at.k[cc]);
        part[cc] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) part[cc] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], __uint_as_float(qf[cc][e]), part[cc], 0, 0, 0);
      }
      return acc + branch<0, NC>(part);
    }
  }
  __device__ __forceinline__ bool take_keys(const Places& at, const char* tile, int j0, const SeqKeys& keys, bool hole, float (&p)[kProbs]) {
    float x[kProbs];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
      if (biased) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = w * (float)max(pos - j0 - key_of(4 * b + e), 0);
      }
      acc = scores(at, tile, b, acc);
      if constexpr (CAP) this->template cap_all<4>(acc, [&](int e) { return pos - j0 - key_of(4 * b + e); });
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * b + e] = acc[e];
    }
    const bool masked = hole || j0 + 32 > lim_min;
    if (masked) {
#pragma unroll
      for (int e = 0; e < kProbs; ++e) {
        const int j = j0 + key_of(e);
        const bool seen = j < lim && !(hole && keys.is_hole(keys.page(j)));
        x[e] = seen ? x[e] : -kInf;
      }
    }
    float m = x[0];
#pragma unroll
    for (int e = 1; e < kProbs; ++e) m = fmaxf(m, x[e]);
    m = other_half_max(fmaxf(m, __shfl_xor(m, 16)));
    const bool more = m > top;  // (as SoftmaxRows::raise)
    if (__ballot(more) != 0ull) {
      const float to = m + this->slack, f = more ? __builtin_amdgcn_exp2f((top - to) * this->unit) : 1.f;
      top = more ? to : top;
      sum *= f;
#pragma unroll
      for (int c4 = 0; c4 < kChunks; ++c4)
#pragma unroll
        for (int e = 0; e < 4; ++e) oacc[c4][e] *= f;
    }
    const float base = top > -kInf ? -top * this->unit : 0.f;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kProbs; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(x[e], this->unit, base));
      s += p[e];
    }
    sum += s;
    return masked;
  }
  // a value of the tile
  static __device__ __forceinline__ float value(const char* tile, int key, int feature) {
    constexpr int E = 16 / (int)sizeof(T);
    const char* at = tile + VTile::off(key, feature / E) + (feature % E) * (int)sizeof(T);
    if constexpr (sizeof(T) == 2)
      return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16);
    else
      return *reinterpret_cast<const float*>(at);
  }
  // oacc += V^T P^T; as in SeqValues::accumulate() where some row does not see some key
  __device__ __forceinline__ void take_values(const Places& at, const char* tile, const float (&p)[kProbs], bool masked) {
    if (masked) {
      bool bad = false;  // (of the tile's bytes as they lie there; one value after the other took 4 us)
#pragma unroll
      for (int e = 0; e < VTile::kBytes / 1024; ++e) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(tile + 1024 * e + 16 * lane);
#pragma unroll
        for (int k = 0; k < 4; ++k) bad = bad || (x[k] & 0x7f800000u) == 0x7f800000u || (sizeof(T) == 2 && (x[k] & 0x7f80u) == 0x7f80u);
      }
      if (__ballot(bad) != 0ull) {
        one_by_one(tile, p);
        return;
      }
    }
    if constexpr (sizeof(T) == 2) {
      // (probabilities as the sum of two bf16 numbers: rounded to one, they would cost up to 2^-9 |v| of the output)
      Frag<T> hi, lo;
      split_pairs(p, hi, lo);
#pragma unroll
      for (int f = 0; f < kChunks; ++f) {
        const uint2 x = read_transposed(tile + at.v[f]), y = read_transposed(tile + at.v[f] + 16 * VTile::kRowBytes);
        const bf16x8_t v = __builtin_bit_cast(bf16x8_t, u32x4_t{x.x, x.y, y.x, y.y});
        oacc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, hi.v), oacc[f], 0, 0, 0);
        oacc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, lo.v), oacc[f], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kProbs; ++e)
#pragma unroll
        for (int f = 0; f < kChunks; ++f) oacc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(value(tile, key_of(e), 16 * f + li), p[e], oacc[f], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void one_by_one(const char* tile, const float (&p)[kProbs]) {
#pragma unroll 1
    for (int from = 0; from < 4; ++from) {
#pragma unroll
      for (int e = 0; e < kProbs; ++e) {
        const float pk = __shfl(p[e], li + 16 * from);
        if (pk > 0.f) {
          const int key = 16 * (e >> 2) + 4 * from + (e & 3);
#pragma unroll
          for (int f = 0; f < kChunks; ++f)
#pragma unroll
            for (int x = 0; x < 4; ++x) oacc[f][x] = fmaf(pk, value(tile, key, 16 * f + 4 * quad + x), oacc[f][x]);
        }
      }
    }
  }
};

// Waves of a workgroup of the kernel that splits the keys, and tiles of 32 keys and values that a wave has in LDS: 64 KB a workgroup, so that two share a
// compute unit and one's start and end hide behind the other's loads.
template <typename T, int D>
struct SoftmaxSplitCfg {
  static constexpr int NW = kSoftmaxWaves<(int)sizeof(T), D>;
  static constexpr int ST = sizeof(T) == 2 && D == 64 ? 2 : 1;
  static constexpr int kTileBytes = 32 * D * (int)sizeof(T);
  static constexpr int kWaveBytes = 2 * ST * kTileBytes;
  static constexpr size_t kLdsBytes = (size_t)NW * kWaveBytes;
};

// A workgroup's piece: place `place`, of sequence v, cut up as sh says.  Rows: SoftmaxRows or SoftmaxRows16; NQB: blocks of them, from row rbase on
template <typename T, int D, class Rows, int NQB>
__device__ __forceinline__ void softmax_split_piece(const SoftmaxArgs& A, int place, int rbase, const SeqView& v, const SoftmaxShare& sh) {
  using Cfg = SoftmaxSplitCfg<T, D>;
  constexpr int NW = Cfg::NW, ST = Cfg::ST, TB = Cfg::kTileBytes, RB = Rows::kRows, CH = Rows::kChunks;
  using KTile = typename Rows::KTile;
  using VTile = typename Rows::VTile;
  constexpr int LD = KTile::L;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float tops[NW][NQB * RB], parts[NW][NQB * RB];
  const SeqGeom& g = A.g;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hk = place % g.Hkv;
  const int split = place / g.Hkv - sh.first;
  if (split >= sh.n) return;
  const int from = split * sh.len, to = min(v.L, from + sh.len);
  const int R = v.n * g.G - rbase;  // rows from there on
  if (R <= 0) return;
  if (A.shared && A.shares && split == 0 && hk == 0 && rbase == 0 && tid == 0) A.shares[v.s] = make_int2(sh.first, sh.n);
  SeqKeys keys, vals;
  keys.init(g, v, A.K, hk, false, sizeof(T));
  vals.init(g, v, A.V, hk, true, sizeof(T));
  char* mine = smem + wave * Cfg::kWaveBytes;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
  // this wave's tiles: from + 32 (wave + NW i); tile i lies in place i % ST
  const int tiles = (to - from + 31) >> 5, nt = tiles > wave ? (tiles - wave + NW - 1) / NW : 0;
  auto start = [&](int i) { return from + 32 * (wave + NW * i); };
  typename KTile::Pages pk;
  typename VTile::Pages pv;
  bool holes[ST];
  auto ask = [&](int i) {
    pk.ask(keys, start(i), v.L, 0);
    pv.ask(vals, start(i), v.L, 0);
  };
  auto issue_k = [&](int i) {
    bool h = false;
#pragma unroll
    for (int it = 0; it < LD; ++it) h = h || keys.is_hole(pk.pg[it]);
    holes[i % ST] = h;
    KTile::load(keys, pk, start(i), v.L, lds + (uint32_t)(2 * (i % ST)) * TB, 0, lane);
  };
  auto issue_v = [&](int i) { VTile::load(vals, pv, start(i), v.L, lds + (uint32_t)(2 * (i % ST) + 1) * TB, 0, lane); };
#pragma unroll
  for (int i = 0; i < ST; ++i) {
    holes[i] = false;
    if (i < nt) {
      ask(i);
      issue_k(i);
      issue_v(i);
    }
  }
  if (nt > ST) ask(ST);
  Rows q[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) q[qb].init(A, v, hk, rbase + qb * RB);
  typename Rows::Places places;
  places.init(lane);
  // A tile's keys, then its values, are waited for; the loads issued after them stay under way: those of the ST - 1 next tiles, and in between the
  // values of this one or the keys of the one that takes its place.
  for (int i = 0; i < nt; ++i) {
    const int left = nt - 1 - i, j0 = start(i);
    const char* tile = mine + 2 * (i % ST) * TB;
    if (ST > 1 && left >= ST - 1)
      lds_loads_wait<(2 * ST - 1) * LD>();
    else
      lds_loads_wait<LD>();
    float p[NQB][Rows::kProbs];
    bool masked[NQB], sees[NQB];
    const bool hole = holes[i % ST];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      sees[qb] = qb * RB < R && j0 < q[qb].lim_max;
      if (sees[qb]) masked[qb] = q[qb].take_keys(places, tile, j0, keys, hole, p[qb]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the keys have been read)
    const bool next = left >= ST;
    if (next) issue_k(i + ST);
    if (next)
      lds_loads_wait<(2 * ST - 1) * LD>();
    else if (ST > 1 && left > 0)
      lds_loads_wait<2 * (ST - 1) * LD>();
    else
      lds_loads_wait<0>();
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
      if (sees[qb]) q[qb].take_values(places, tile + TB, p[qb], masked[qb]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (next) issue_v(i + ST);
    if (left > ST) ask(i + ST + 1);
  }
  // the waves' outputs in units of their largest score, added in their order
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const float l = q[qb].total();
    if (q[qb].first_lane()) {
      tops[wave][qb * RB + q[qb].row()] = q[qb].top2();
      parts[wave][qb * RB + q[qb].row()] = l;
    }
  }
  __syncthreads();  // (no tile is read any more)
  const int pieces = sh.n;
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    if (qb * RB >= R) break;
    const int row = qb * RB + q[qb].row();
    float most = -kInf, l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) most = fmaxf(most, tops[w][row]);
    auto factor = [&](int w) { return most > -kInf ? __builtin_amdgcn_exp2f(tops[w][row] - most) : 0.f; };
#pragma unroll
    for (int w = 0; w < NW; ++w) l += parts[w][row] * factor(w);
    const float f = factor(wave);
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);  // [waves][CH][64]
    static_assert(CH * 1024 <= Cfg::kWaveBytes, "a wave's outputs fit its tiles");
    if (qb) __syncthreads();
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      f32x4_t o = q[qb].out(u);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= f;
      red[(wave * CH + u) * 64 + lane] = o;
    }
    __syncthreads();
    const float inv = l > 0.f ? 1.f / l : 0.f;
    for (int u = wave; u < CH; u += NW) {
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const f32x4_t x = red[(w * CH + u) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[e];
      }
      if (row >= R) continue;
      const int feature = q[qb].feature(u);
      if (pieces > 1) {
        *reinterpret_cast<f32x4_t*>(A.part + ((long long)place * A.rows + rbase + row) * D + feature) = o;
      } else {
        T* dst = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + q[qb].t) * g.o_st + (long long)q[qb].head * g.o_sh + feature;
        store4<T>(dst, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
      }
    }
    if (wave == 0 && q[qb].first_lane() && row < R) {
      if (pieces > 1)
        A.sums[(long long)place * A.rows + rbase + row] = make_float2(most, l);
      else if (A.lse)
        A.lse[(long long)q[qb].head * g.T + v.row0 + q[qb].t] = l > 0.f ? (most + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
    }
  }
}

template <typename T, int D, class Rows, int NQB>
__global__ __launch_bounds__((SoftmaxSplitCfg<T, D>::NW * 64), (NQB == 1 && (sizeof(T) == 2 || Rows::kRows == 16) ? 2 : 1)) void softmax_split_kernel(
    SoftmaxArgs A) {
  SeqView v;
  SoftmaxShare sh;
  if (softmax_share(A, (int)blockIdx.x / A.g.Hkv, v, sh)) softmax_split_piece<T, D, Rows, NQB>(A, blockIdx.x, blockIdx.z * NQB * Rows::kRows, v, sh);
}

// Adds up the pieces of a row: piece k's output at part + k step D, its (largest score, sum) at sums[k step].  `slices` groups of D / 4 threads share them, each
// thread with four features; what they have found meets in LDS.  f: this thread's first feature; slice 0's threads end with the row's output and lse.
template <int D>
struct SoftmaxJoin {
  static constexpr int LR = D / 4;
  f32x4_t outs[kThreads];
  float2 found[kThreads / LR];
  __device__ __forceinline__ float add_up(const float* part, const float2* sums, int pieces, long long step, int slice, int slices, int f, f32x4_t& o) {
    const int tid = threadIdx.x, group = tid / LR;
    float most = -kInf, l = 0.f;
    o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = slice; k < pieces; k += slices) most = fmaxf(most, sums[k * step].x);
#pragma unroll 8
    for (int k = slice; k < pieces; k += slices) {
      const float2 x = sums[k * step];
      const f32x4_t y = *reinterpret_cast<const f32x4_t*>(part + k * step * D + f);
      const float w = x.y > 0.f ? __builtin_amdgcn_exp2f(x.x - most) : 0.f;
      l = fmaf(x.y, w, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], w, o[e]);
    }
    if (slices > 1) {
      outs[tid] = o;
      if (f == 0) found[group] = make_float2(most, l);
      __syncthreads();
      if (slice != 0) return 0.f;
      for (int k = 0; k < slices; ++k) most = fmaxf(most, found[group + k].x);
      l = 0.f;
      o = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < slices; ++k) {
        const float2 x = found[group + k];
        const float w = x.y > 0.f ? __builtin_amdgcn_exp2f(x.x - most) : 0.f;
        l = fmaf(x.y, w, l);
        const f32x4_t y = outs[tid + k * LR];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], w, o[e]);
      }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    return l > 0.f ? (most + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
  }
};

template <typename T, int D>
__device__ __forceinline__ void store_joined(const SoftmaxArgs& A, const SeqView& v, int hk, int row, int f, const f32x4_t& o, float lse) {
  const SeqGeom& g = A.g;
  const int t = row / g.G, qh = hk * g.G + row - t * g.G;
  T* dst = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + t) * g.o_st + (long long)qh * g.o_sh + f;
  store4<T>(dst, o[0], o[1], o[2], o[3]);
  if (f == 0 && A.lse) A.lse[(long long)qh * g.T + v.row0 + t] = lse;
}

// Both kinds of pieces: workgroups 0 .. tiled - 1 for those of groups, kThreads / (D / 4) rows each, the others for those of softmax_split_piece()
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void softmax_join_kernel(SoftmaxArgs A, int tiled, int slices) {
  using Join = SoftmaxJoin<D>;
  __shared__ Join join;
  const SeqGeom& g = A.g;
  const int tid = threadIdx.x, group = tid / Join::LR, f = (tid % Join::LR) * 4, hk = blockIdx.x % g.Hkv;
  SeqView v;
  SoftmaxShare sh;
  f32x4_t o;
  if ((int)blockIdx.x < tiled) {
    constexpr int RW = kThreads / Join::LR, PER = kBlockRows / RW;
    const int x = (int)blockIdx.x / g.Hkv, blk = x / PER;
    int blk0;
    if (!seq_block(g, blk, A.split != 0, v, blk0)) return;
    const int local = x % PER * RW + group, row = blk0 + local, last_row = min(v.n * g.G, blk0 + kBlockRows) - 1;
    sh.cut(g.causal ? max(0, min(v.L - v.n + last_row / g.G + 1, v.L)) : v.L, A.tpiece >> 5, 2);
    if (sh.n <= 1 || row > last_row) return;
    const long long at = ((long long)blk * g.Hkv + hk) * A.tsplits * kBlockRows + local;
    const float lse = join.add_up(A.tpart + at * D, A.tsums + at, sh.n, kBlockRows, 0, 1, f, o);
    store_joined<T, D>(A, v, hk, row, f, o, lse);
    return;
  }
  const int x = ((int)blockIdx.x - tiled) / g.Hkv, per_wg = kThreads / (Join::LR * slices), per = (A.rows + per_wg - 1) / per_wg;
  const int s = x / per, slice = group % slices, row0 = x % per * per_wg, row = row0 + group / slices;
  if (!load_seq(g, s, v) || !split_seq(g, v) || row0 >= v.n * g.G) return;
  if (A.shared) {
    const int2 share = A.shares[s];
    sh.first = share.x;
    sh.n = share.y;
  } else {
    sh.cut(v.L, A.piece >> 5);
    sh.first = s * A.splits;
  }
  if (sh.n <= 1) return;  // (the same for the workgroup)
  const bool mine = row < v.n * g.G;
  const long long at = ((long long)sh.first * g.Hkv + hk) * A.rows + (mine ? row : 0);
  const float lse = join.add_up(A.part + at * D, A.sums + at, sh.n, (long long)g.Hkv * A.rows, slice, slices, f, o);
  if (mine && slice == 0) store_joined<T, D>(A, v, hk, row, f, o, lse);
}

template <typename T, int D>
struct SoftmaxTiledCfg {
  static constexpr int KT = sizeof(T) == 4 && D == 128 ? 32 : 64;
  static constexpr int kTileBytes = KT * D * (int)sizeof(T);
  static constexpr size_t kLdsBytes = 4 * (size_t)kTileBytes;
  static constexpr int kWavesPerSimd = sizeof(T) == 4 && D == 128 ? 1 : 2;
  static constexpr int NB = sizeof(T) == 2 ? 2 : 1;  // blocks of 32 keys that a wave takes in together
};

// The two waves of a SIMD hide each other's exponentials and LDS reads behind their products; what counts is how much else a tile costs.  bf16, 16 x 512 tokens
// against 2048 keys, 4 x 4 heads of 128: 308 us (447 TFLOP/s) with the address of every load from its page and limit and a rescaling of the sums inside the loop (32 register
// pairs copied a tile), 263 without, 200 with a `top` that is left for good after a few tiles.  4096 tokens against themselves, 16 heads: 139 us (495 TFLOP/s of the pairs
// that rows see, half of all; with the product of V made twice 740 are done).
template <typename T, int D, bool CAP>
__device__ __forceinline__ void softmax_tiled_piece(const SoftmaxArgs& A, int wg) {
  using Cfg = SoftmaxTiledCfg<T, D>;
  constexpr int KT = Cfg::KT, NB = Cfg::NB, NC = D / 16, NM = D / 32, TB = Cfg::kTileBytes;
  using KTile = SeqTile<T, D, KT, false>;
  using Vals = SeqValues<T, D, KT>;
  using VTile = typename Vals::VT;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const SeqGeom& g = A.g;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // (heads and groups in the order of the entmax attention's tiled kernel; a group's pieces next to each other)
  const int hk = wg % g.Hkv, piece = wg / g.Hkv % A.tsplits, blk = A.nblk - 1 - wg / g.Hkv / A.tsplits;
  SeqView v;
  int blk0;
  if (!seq_block(g, blk, A.split != 0, v, blk0)) return;
  SeqKeys keys, vals;
  keys.init(g, v, A.K, hk, false, sizeof(T));
  vals.init(g, v, A.V, hk, true, sizeof(T));
  SoftmaxRows<T, D, CAP> q;
  q.init(A, v, hk, blk0 + wave * 32);
  const int last_row = min(v.n * g.G, blk0 + kBlockRows) - 1;
  const int block_lim = g.causal ? max(0, min(v.L - v.n + last_row / g.G + 1, v.L)) : v.L;
  SoftmaxShare sh;
  sh.cut(block_lim, A.tpiece >> 5, 2);  // (tiles of 64 keys in all pieces, also where this kernel's are of 32)
  if (piece >= sh.n) return;
  const int key0 = piece * sh.len, ntiles = __builtin_amdgcn_readfirstlane((min(block_lim - key0, sh.len) + KT - 1) / KT);
  const bool holes = seq_has_holes(keys, min(v.L, (block_lim + KT - 1) / KT * KT));  // (whole tiles are loaded, also behind the last key that a row sees)
  const int lane = q.lane;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  FragOff<T> koff[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc) koff[cc] = FragOff<T>::template make<typename KTile::Tile>(q.li, 2 * cc + q.hh);
  Vals vv;
  vv.init(lane);
  // bf16: the first `plain` tiles have no key that some row of the workgroup does not see (limits do not decrease from row to row)
  bool whole = NB == 2 && !holes && keys.sp >> 32 == 0 && vals.sp >> 32 == 0 && (keys.sn << g.lps) >> 31 == 0 && (vals.sn << g.lps) >> 31 == 0;
  whole = __builtin_amdgcn_readfirstlane(whole ? 1 : 0) != 0;
  int plain = 0;
  if constexpr (NB == 2) {
    const int first_lim = g.causal ? max(0, min(v.L - v.n + blk0 / g.G + 1, v.L)) : v.L;
    plain = __builtin_amdgcn_readfirstlane(whole ? max(0, min(ntiles, (first_lim - key0) / KT)) : 0);
  }
  // Tiles on their way, their pages asked for one tile ahead (the same for keys and values).  `whole`, and no row behind the last: 32-bit offsets, the same of a
  // lane in all its loads (the swizzle has the period of a load's rows), and nothing to clamp.
  static_assert(VTile::L == KTile::L && VTile::RS == KTile::RS && VTile::RW == KTile::RW && (NB == 1 || KTile::RS % 16 == 0), "loads of the same rows");
  // From the last tile to the first: where the bias or the model prefers near keys, the largest scores come first and `top` stays.  (8 biased heads of 16, 5 sequences of
  // 100 to 187 tokens against 564 to 4930 keys: 69 us from the first, 56 so; without a bias within 3 % of each other.)
  auto key_of = [&](int t) { return key0 + (ntiles - 1 - t) * KT; };
  typename KTile::Pages pages;
  auto ask = [&](int t) {
    pages.ask(keys, key_of(t), v.L, wave);
#pragma unroll
    for (int it = 0; it < KTile::L; ++it) pages.pg[it] = __builtin_amdgcn_readfirstlane(pages.pg[it]);
  };
  const int load_row = wave * KTile::RW + lane / KTile::kCpr;
  const uint32_t klane = (uint32_t)(lane / KTile::kCpr) * (uint32_t)keys.sn + (uint32_t)(((lane % KTile::kCpr) ^ KTile::swz(load_row)) << 4);
  const uint32_t vlane = (uint32_t)(lane / VTile::kCpr) * (uint32_t)vals.sn + (uint32_t)(((lane % VTile::kCpr) ^ VTile::swz(load_row)) << 4);
  auto issue = [&](int t, int buf) {
    const uint32_t kdst = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)(2 * buf) * TB), vdst = kdst + TB;
    if (NB == 2 && whole && key_of(t) + KT <= v.L) {
      const uint32_t mask = (1u << g.lps) - 1u;
#pragma unroll
      for (int it = 0; it < KTile::L; ++it) {
        const uint32_t at = (uint32_t)(key_of(t) + it * KTile::RS + wave * KTile::RW) & mask, dst = (uint32_t)((it * kThreads + wave * 64) * 16);
        const uint32_t pg = (uint32_t)pages.pg[it];
        load_to_lds(uniform(keys.base + ((unsigned long long)pg * (uint32_t)keys.sp + at * (uint32_t)keys.sn)), klane, kdst + dst);
        load_to_lds(uniform(vals.base + ((unsigned long long)pg * (uint32_t)vals.sp + at * (uint32_t)vals.sn)), vlane, vdst + dst);
      }
    } else {
      typename VTile::Pages same;
#pragma unroll
      for (int it = 0; it < KTile::L; ++it) same.pg[it] = pages.pg[it];
      KTile::load(keys, pages, key_of(t), v.L, kdst, wave, lane);
      VTile::load(vals, same, key_of(t), v.L, vdst, wave, lane);
    }
  };
  if (ntiles > 0) {
    ask(0);
    issue(0, 0);
  }
  if (ntiles > 1) ask(1);
  lds_loads_wait<0>();
  __syncthreads();
  // Every wave meets the others once a tile, in the first loop or in what follows it.
  int t = 0;
  while (t < ntiles) {
    bool ahead = false;  // of the loads of the next tile
    if constexpr (NB == 2) {
      // as long as no row's largest score goes up by much: nothing here rescales the sums, so they stay in their registers
#pragma unroll 1
      for (; t >= ntiles - plain && t < ntiles; ++t) {
        if (t + 1 < ntiles) {
          issue(t + 1, (t + 1) & 1);
          if (t + 2 < ntiles) ask(t + 2);
        }
        const char* tile = smem + (t & 1) * 2 * TB;
        f32x16_t acc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
          acc[b] = CAP ? q.start(key_of(t) + 32 * b) : f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int cc = 0; cc < NC; ++cc)  // (two sums in turn: neither waits for its last product)
#pragma unroll
          for (int b = 0; b < 2; ++b) acc[b] = Elem<T>::mma(koff[cc].load(tile, b * 32 * KTile::kRowBytes), q.qf[cc], acc[b]);
        Frag<T> vf[2][NM];
        auto fetch = [&](int u) {  // values of the 16 keys 16 u .. of the tile
#pragma unroll
          for (int mm = 0; mm < NM; ++mm) vf[u & 1][mm] = vv.frag(tile + TB, u >> 1, u & 1, mm);
        };
        fetch(0);
        if (!CAP && q.biased) {  // (afterwards: a start for it would be 32 registers to clear in each tile; with a cap they do not count and the code would spill)
#pragma unroll
          for (int b = 0; b < 2; ++b) q.add_bias(acc[b], key_of(t) + 32 * b);
        }
        if constexpr (CAP) {
#pragma unroll
          for (int b = 0; b < 2; ++b) q.cap_scores(acc[b], key_of(t) + 32 * b);
        }
        if (q.template rises<2>(acc)) {
          ahead = true;
          break;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (u + 1 < 4) fetch(u + 1);
          float p[8];
          q.probs8(acc[u >> 1], 8 * (u & 1), p);
          // the probabilities as the sum of two bf16 numbers: rounded to one, they would cost up to 2^-9 |v| of the output (and save a seventh of the time)
          Frag<T> hi, lo;
          split_pairs(p, hi, lo);
#pragma unroll
          for (int mm = 0; mm < NM; ++mm) q.oacc[mm] = Elem<T>::mma(vf[u & 1][mm], hi, q.oacc[mm]);
#pragma unroll
          for (int mm = 0; mm < NM; ++mm) q.oacc[mm] = Elem<T>::mma(vf[u & 1][mm], lo, q.oacc[mm]);
        }
        lds_loads_wait<0>();
        __syncthreads();
      }
      if (t >= ntiles) break;
    }
    if (!ahead && t + 1 < ntiles) {
      issue(t + 1, (t + 1) & 1);
      if (t + 2 < ntiles) ask(t + 2);
    }
    const char* tile = smem + (t & 1) * 2 * TB;
#pragma unroll 1
    for (int sb = 0; sb < KT / 32; ++sb) {
      const int j0 = key_of(t) + sb * 32;
      if (j0 >= q.lim_max) break;
      const char* at = tile + sb * 32 * KTile::kRowBytes;
      f32x16_t acc[1] = {q.scores(q.start(j0), [&](int cc) { return koff[cc].load(at, 0); })};
      if constexpr (CAP) q.cap_scores(acc[0], j0);
      const bool masked = holes || j0 + 32 > q.lim_min;
      if (masked) q.mask(acc[0], j0, keys, holes);
      q.template raise<1>(acc);
      float p[16];
      q.probs(acc[0], p);
      vv.accumulate(tile + TB, sb, p, masked, q.oacc);
    }
    lds_loads_wait<0>();
    __syncthreads();
    ++t;
  }
  const float l = q.total();
  if (!q.valid) return;
  if (sh.n > 1) {
    const long long at = (((long long)blk * g.Hkv + hk) * A.tsplits + piece) * kBlockRows + wave * 32 + q.li;
#pragma unroll
    for (int u = 0; u < q.kChunks; ++u) *reinterpret_cast<f32x4_t*>(A.tpart + at * D + q.feature(u)) = q.out(u);
    if (q.hh == 0) A.tsums[at] = make_float2(q.top2(), l);
    return;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T* o = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + q.t) * g.o_st + (long long)q.head * g.o_sh;
#pragma unroll
  for (int mm = 0; mm < NM; ++mm)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      store4<T>(o + 32 * mm + 8 * x + 4 * q.hh, q.oacc[mm][4 * x] * inv, q.oacc[mm][4 * x + 1] * inv, q.oacc[mm][4 * x + 2] * inv,
                q.oacc[mm][4 * x + 3] * inv);
  if (A.lse && q.hh == 0) A.lse[(long long)q.head * g.T + v.row0 + q.t] = l > 0.f ? (q.top2() + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
}

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(kThreads, (SoftmaxTiledCfg<T, D>::kWavesPerSimd)) void softmax_tiled_kernel(SoftmaxArgs A) {
  softmax_tiled_piece<T, D, CAP>(A, blockIdx.x);
}

// Prompts and sequences of few rows in one call, at the same time: workgroups 0 .. tiled - 1 for the groups, the others for the pieces.  (bf16, whose two
// kinds of workgroups are of one size.  18 sequences of one token and one of 20 against up to
// 4355 keys, 4 x 4 heads of 128, capped and biased: 92 us one after the other, 42 so.)
template <typename T, int D, bool CAP>
__global__ __launch_bounds__(kThreads, (SoftmaxTiledCfg<T, D>::kWavesPerSimd)) void softmax_mixed_kernel(SoftmaxArgs A, int tiled) {
  static_assert(SoftmaxSplitCfg<T, D>::NW * 64 == kThreads, "one size of workgroups");
  if ((int)blockIdx.x < tiled) {
    softmax_tiled_piece<T, D, CAP>(A, blockIdx.x);
    return;
  }
  const int place = (int)blockIdx.x - tiled;
  SeqView v;
  SoftmaxShare sh;
  if (!softmax_share(A, place / A.g.Hkv, v, sh)) return;
  if (v.n * A.g.G <= 16)
    softmax_split_piece<T, D, SoftmaxRows16<T, D, CAP>, 1>(A, place, 0, v, sh);
  else {
    constexpr int NQB = D == 64 ? 2 : 1;  // (two blocks of 128 features leave no room for a second workgroup on the compute unit)
#pragma unroll 1
    for (int rbase = 0; rbase < v.n * A.g.G; rbase += 32 * NQB) {
      if (rbase) __syncthreads();  // (what the last ones left in LDS has been read)
      softmax_split_piece<T, D, SoftmaxRows<T, D, CAP>, NQB>(A, place, rbase, v, sh);
    }
  }
}

// Enqueues the call for checked parameters; returns an entmax_attn_status.
template <typename T, int D>
int run_softmax(const SoftmaxCall& c);

namespace {

template <typename T, int D, class Rows, int NQB>
bool launch_softmax_split(const SoftmaxArgs& a, long long places, hipStream_t st) {
  using Cfg = SoftmaxSplitCfg<T, D>;
  constexpr auto kern = softmax_split_kernel<T, D, Rows, NQB>;
  if (!ensure_dynamic_lds<kern>(Cfg::kLdsBytes)) return false;
  const dim3 grid((unsigned)places, 1, (unsigned)ceil_div(a.rows, NQB * Rows::kRows));
  hipLaunchKernelGGL(kern, grid, dim3(Cfg::NW * 64), Cfg::kLdsBytes, st, a);
  return launch_ok();
}

template <typename T, int D, bool CAP>
bool launch_softmax(const SoftmaxArgs& a, const SoftmaxLayout& L, hipStream_t st) {
  using Tiled = SoftmaxTiledCfg<T, D>;
  const unsigned groups = (unsigned)(a.nblk * a.g.Hkv), tiled = L.blocks ? groups * (unsigned)a.tsplits : 0u;
  bool split = L.split;
  if (L.blocks) {
    if constexpr (sizeof(T) == 2) {
      if (split) {
        constexpr auto kern = softmax_mixed_kernel<T, D, CAP>;
        constexpr size_t lds = Tiled::kLdsBytes > SoftmaxSplitCfg<T, D>::kLdsBytes ? Tiled::kLdsBytes : SoftmaxSplitCfg<T, D>::kLdsBytes;
        if (!ensure_dynamic_lds<kern>(lds)) return false;
        hipLaunchKernelGGL(kern, dim3(tiled + (unsigned)L.places), dim3(kThreads), lds, st, a, (int)tiled);
        if (!launch_ok()) return false;
      }
    }
    if (sizeof(T) == 4 || !split) {
      constexpr auto kern = softmax_tiled_kernel<T, D, CAP>;
      if (!ensure_dynamic_lds<kern>(Tiled::kLdsBytes)) return false;
      hipLaunchKernelGGL(kern, dim3(tiled), dim3(kThreads), Tiled::kLdsBytes, st, a);
      if (!launch_ok()) return false;
    }
    if (sizeof(T) == 2) split = false;  // (done)
  }
  if (split) {
    // (two blocks of fp32 rows of 128 features do not fit the registers)
    constexpr int kMostBlocks = sizeof(T) == 4 && D == 128 ? 1 : 2;
    const bool ok = a.rows <= 16   ? launch_softmax_split<T, D, SoftmaxRows16<T, D, CAP>, 1>(a, L.places, st)
                    : a.rows <= 32 ? launch_softmax_split<T, D, SoftmaxRows<T, D, CAP>, 1>(a, L.places, st)
                                   : launch_softmax_split<T, D, SoftmaxRows<T, D, CAP>, kMostBlocks>(a, L.places, st);
    if (!ok) return false;
  }
  const unsigned of_groups = L.blocks && a.tsplits > 1 ? groups * (unsigned)(kBlockRows * D / 4 / kThreads) : 0u;
  unsigned of_pieces = 0;
  int slices = 1;  // (a power of two: two pieces or more to each)
  if (L.split && L.most_pieces > 1) {
    while (2 * slices <= kThreads / (D / 4) && 4 * slices <= L.most_pieces) slices *= 2;
    of_pieces = (unsigned)(a.g.nseq * a.g.Hkv) * (unsigned)ceil_div(a.rows, kThreads / (D / 4) / slices);
  }
  if (of_groups + of_pieces == 0) return true;
  hipLaunchKernelGGL((softmax_join_kernel<T, D>), dim3(of_groups + of_pieces), dim3(kThreads), 0, st, a, (int)of_groups, slices);
  return launch_ok();
}

}  // namespace

template <typename T, int D>
int run_softmax(const SoftmaxCall& c) {
  const entmax_seq_params* p = c.p;
  const SoftmaxLayout L = make_softmax_layout(p);
  SoftmaxArgs a;
  a.g = SeqGeom{p->nseq, p->T, p->Hq, p->Hkv, p->Hq / p->Hkv, p->causal, p->scale_layout, p->logn_mode, p->bias_mode, 2.0f, p->delta, c.beta, c.gamma,
                c.slopes, c.cu, c.kv_len, c.table, __builtin_ctz((unsigned)p->page_size), p->num_pages, p->max_pages, p->max_new, p->max_keys,
                p->q_stride_t, p->q_stride_h, p->o_stride_t, p->o_stride_h, p->k_stride_p, p->k_stride_h, p->k_stride_n, p->v_stride_p, p->v_stride_h,
                p->v_stride_n};
  a.Q = c.Q;
  a.K = c.K;
  a.V = c.V;
  a.O = c.O;
  a.lse = c.lse;
  a.cap = c.cap;
  a.part = reinterpret_cast<float*>(c.ws + L.off_part);
  a.sums = reinterpret_cast<float2*>(c.ws + L.off_sums);
  a.shares = L.most_pieces > 1 ? reinterpret_cast<int2*>(c.ws + L.off_shares) : nullptr;
  a.rows = L.rows;
  a.shared = L.shared ? 1 : 0;
  a.budget = L.budget;
  a.least = L.least;
  a.piece = L.piece;
  a.splits = L.splits;
  a.nblk = (int)seq_blocks(p->nseq, p->T, a.g.G);
  a.split = L.split ? 1 : 0;
  a.tpart = reinterpret_cast<float*>(c.ws + L.off_tpart);
  a.tsums = reinterpret_cast<float2*>(c.ws + L.off_tsums);
  a.tpiece = L.tpiece;
  a.tsplits = L.tsplits;
  const bool ok = c.cap > 0.f && c.cap <= kSoftmaxMostCap ? launch_softmax<T, D, true>(a, L, c.st) : launch_softmax<T, D, false>(a, L, c.st);
  return ok ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // namespace entmax
