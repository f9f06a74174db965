// Softmax attention of new tokens over a paged cache: o_i = sum_j p_ij v_j, p_ij = exp(s_ij - lse_i), with the scales, bias and masks of the entmax
// attention and, if asked for, scores capped by a tanh.  One pass over keys and values: a row's largest score and sum so far, its output so far
// scaled down whenever a larger score comes.  Scores as in the tiled kernel there, S^T = K Q^T with a lane pair for each of 32 folded rows (token, head of the
// group), whose probabilities are the second operand of O^T = V^T P^T as they are.
//   softmax_split_kernel  sequences of at most kSplitRows folded rows (decode steps): the keys are cut into pieces, a workgroup each.  A wave
//                         goes through 32-key tiles of its own, brought to LDS by loads that it alone waits for; the waves meet at the end.
//                         Bound by the one read of K and V.
//   softmax_join_kernel   adds up the pieces' outputs, each in units of its own largest score
//   softmax_tiled_kernel  others: a workgroup per 128 folded rows, tiles of keys and values shared by its waves
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
  float* part;    // [nseq * Hkv][splits][rows][D]
  float2* sums;   // [nseq * Hkv][splits][rows] (largest score in units of log 2, sum)
  int rows, piece, splits;
  int nblk;
  int split;      // sequences with few rows are left to softmax_split_kernel
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A row's scores in units of log 2, and what it has seen so far.
template <typename T, int D, bool CAP>
struct SoftmaxRows : SeqRows<T, D> {
  static constexpr int NM = D / 32;
  float unit;        // score = unit * accumulator
  float cap2, in2;   // CAP: cap in units of log 2; the accumulator's factor in exp2(2 s / cap)
  float late;        // CAP, bias outside the cap: its slope
  float top, sum;    // largest accumulator; sum of this lane's exp2(unit (acc - top))
  f32x16_t oacc[NM];
  __device__ __forceinline__ void init(const SoftmaxArgs& A, const SeqView& v, int hk, int r0) {
    SeqRows<T, D>::init(A.g, v, A.Q, hk, r0);
    unit = CAP ? 1.f : this->a * kLog2e;
    if (CAP) {
      cap2 = A.cap * kLog2e;
      in2 = this->a / A.cap;
      late = 0.f;
      if (A.g.bias_mode == 1) {
        late = this->a * this->w * kLog2e;
        this->w = 0.f;
        this->biased = false;
      }
    }
    top = -kInf;
    sum = 0.f;
#pragma unroll
    for (int mm = 0; mm < NM; ++mm)
      oacc[mm] = f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  }
  // S^T of 32 keys as in SeqRows; fp32: sums of sixteen features each, one after the other so that few of them are held, added up as a tree
  template <class F>
  __device__ __forceinline__ f32x16_t scores(f32x16_t acc, F frag) const {
    if constexpr (sizeof(T) == 2) return this->dots(acc, frag);
    else return acc + branch<0, D / 16>(frag);
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
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float t;
      if constexpr (sizeof(T) == 2)  // (1.2e-7 of the cap off: far below what rounding Q and K costs)
        t = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(acc[e] * (2.f * kLog2e * in2)));
      else
        t = tanhf(acc[e] * in2);
      acc[e] = fmaf(late, (float)max(this->pos - j0 - this->key_of(e), 0), cap2 * t);
    }
  }
  // Takes in the 32 keys from j0 on, whose scores' accumulators acc are (masked ones -inf): p receives exp2(score - largest so far)
  __device__ __forceinline__ void step(const f32x16_t& acc, float (&p)[16]) {
    float m = max16(acc);
    m = fmaxf(m, __shfl_xor(m, 32));
    const bool more = m > top;
    if (__ballot(more) != 0ull) {
      const float f = more ? __builtin_amdgcn_exp2f((top - m) * unit) : 1.f;  // (0 from -inf)
      top = more ? m : top;
      sum *= f;
#pragma unroll
      for (int mm = 0; mm < NM; ++mm)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[mm][e] *= f;
    }
    const float base = top > -kInf ? -top * unit : 0.f;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(acc[e], unit, base));
      s += p[e];
    }
    sum += s;
  }
  __device__ __forceinline__ float top2() const { return top > -kInf ? top * unit : -kInf; }
};

template <typename T, int D>
struct SoftmaxSplitCfg {
  static constexpr int NW = sizeof(T) == 4 && D == 128 ? 2 : 4;
  static constexpr int KT = 32, kTileBytes = KT * D * (int)sizeof(T);
  static constexpr int kWaveBytes = 4 * kTileBytes;  // two tiles of keys, two of values
  static constexpr size_t kLdsBytes = (size_t)NW * kWaveBytes;
};

template <typename T, int D, int NQB, bool CAP>
__global__ __launch_bounds__((SoftmaxSplitCfg<T, D>::NW * 64), 1) void softmax_split_kernel(SoftmaxArgs A) {
  using Cfg = SoftmaxSplitCfg<T, D>;
  constexpr int NW = Cfg::NW, NC = D / 16, NM = D / 32, TB = Cfg::kTileBytes;
  using KTile = SeqTile<T, D, 32, false, 64>;
  using Vals = SeqValues<T, D, 32, 64>;
  using VTile = typename Vals::VT;
  constexpr int LD = KTile::L;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float tops[NW][NQB * 32], parts[NW][NQB * 32];
  const SeqGeom& g = A.g;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, li = lane & 31, hh = lane >> 5;
  const int split = blockIdx.x % A.splits, s = blockIdx.x / A.splits, hk = blockIdx.y;
  SeqView v;
  if (!load_seq(g, s, v) || !split_seq(g, v)) return;
  const int from = split * A.piece;
  if (split > 0 && from >= v.L) return;
  const int to = min(v.L, from + A.piece);
  const int rbase = blockIdx.z * NQB * 32, R = v.n * g.G - rbase;  // first row, rows from there on
  if (R <= 0) return;
  SeqKeys keys, vals;
  keys.init(g, v, A.K, hk, false, sizeof(T));
  vals.init(g, v, A.V, hk, true, sizeof(T));
  char* mine = smem + wave * Cfg::kWaveBytes;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
  // this wave's tiles: from + 32 (wave + NW i)
  const int tiles = (to - from + 31) >> 5, nt = tiles > wave ? (tiles - wave + NW - 1) / NW : 0;
  auto start = [&](int i) { return from + 32 * (wave + NW * i); };
  typename KTile::Pages pk;
  typename VTile::Pages pv;
  bool holes[2] = {false, false};
  auto ask = [&](int i) {
    pk.ask(keys, start(i), v.L, 0);
    pv.ask(vals, start(i), v.L, 0);
  };
  auto issue_k = [&](int i, int buf) {
    bool h = false;
#pragma unroll
    for (int it = 0; it < LD; ++it) h = h || keys.is_hole(pk.pg[it]);
    holes[buf] = h;
    KTile::load(keys, pk, start(i), v.L, lds + (uint32_t)(2 * buf) * TB, 0, lane);
  };
  auto issue_v = [&](int i, int buf) { VTile::load(vals, pv, start(i), v.L, lds + (uint32_t)(2 * buf + 1) * TB, 0, lane); };
  if (nt > 0) {
    ask(0);
    issue_k(0, 0);
    issue_v(0, 0);
  }
  if (nt > 1) {
    ask(1);
    issue_k(1, 1);
    issue_v(1, 1);
  }
  if (nt > 2) ask(2);
  SoftmaxRows<T, D, CAP> q[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) q[qb].init(A, v, hk, rbase + qb * 32);
  FragOff<T> koff[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc) koff[cc] = FragOff<T>::template make<typename KTile::Tile>(li, 2 * cc + hh);
  Vals vv;
  vv.init(lane);
  for (int i = 0; i < nt; ++i) {
    const int buf = i & 1, left = nt - 1 - i, j0 = start(i);
    const char* tile = mine + 2 * buf * TB;
    if (left > 0)
      lds_loads_wait<3 * LD>();
    else
      lds_loads_wait<LD>();
    float p[NQB][16];
    bool masked[NQB], sees[NQB];
    const bool hole = holes[buf];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      sees[qb] = qb * 32 < R && j0 < q[qb].lim_max;
      if (!sees[qb]) continue;
      f32x16_t acc = q[qb].scores(q[qb].start(j0), [&](int cc) { return koff[cc].load(tile, 0); });
      if constexpr (CAP) q[qb].cap_scores(acc, j0);
      masked[qb] = hole || j0 + 32 > q[qb].lim_min;
      if (masked[qb]) q[qb].mask(acc, j0, keys, hole);
      q[qb].step(acc, p[qb]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the tile has been read)
    if (left > 1) issue_k(i + 2, buf);
    if (left > 1)
      lds_loads_wait<3 * LD>();
    else if (left > 0)
      lds_loads_wait<2 * LD>();
    else
      lds_loads_wait<0>();
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
      if (sees[qb]) vv.accumulate(tile + TB, 0, p[qb], masked[qb], q[qb].oacc);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (left > 1) issue_v(i + 2, buf);
    if (left > 2) ask(i + 3);
  }
  // the waves' outputs in units of their largest score, added in their order
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const float l = q[qb].sum + __shfl_xor(q[qb].sum, 32);
    if (hh == 0) {
      tops[wave][qb * 32 + li] = q[qb].top2();
      parts[wave][qb * 32 + li] = l;
    }
  }
  __syncthreads();  // (no tile is read any more)
  const int pieces = max(1, (v.L + A.piece - 1) / A.piece);
  const long long head = (long long)s * g.Hkv + hk;
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    if (qb * 32 >= R) break;
    float most = -kInf, l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) most = fmaxf(most, tops[w][qb * 32 + li]);
    auto factor = [&](int w) { return most > -kInf ? __builtin_amdgcn_exp2f(tops[w][qb * 32 + li] - most) : 0.f; };
#pragma unroll
    for (int w = 0; w < NW; ++w) l += parts[w][qb * 32 + li] * factor(w);
    const float f = factor(wave);
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);  // [waves][NM * 4][64]
    if (qb) __syncthreads();
#pragma unroll
    for (int mm = 0; mm < NM; ++mm)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        f32x4_t o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = q[qb].oacc[mm][4 * x + e] * f;
        red[(wave * NM * 4 + mm * 4 + x) * 64 + lane] = o;
      }
    __syncthreads();
    const int row = qb * 32 + li;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    for (int u = wave; u < NM * 4; u += NW) {  // features 8 u + 4 hh on of this lane's row
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const f32x4_t x = red[(w * NM * 4 + u) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[e];
      }
      if (row >= R) continue;
      if (pieces > 1) {
        *reinterpret_cast<f32x4_t*>(A.part + ((head * A.splits + split) * A.rows + rbase + row) * D + 8 * u + 4 * hh) = o;
      } else {
        T* dst = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + q[qb].t) * g.o_st + (long long)q[qb].head * g.o_sh + 8 * u + 4 * hh;
        store4<T>(dst, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
      }
    }
    if (wave == 0 && hh == 0 && row < R) {
      if (pieces > 1)
        A.sums[(head * A.splits + split) * A.rows + rbase + row] = make_float2(most, l);
      else if (A.lse)
        A.lse[(long long)q[qb].head * g.T + v.row0 + q[qb].t] = l > 0.f ? (most + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
    }
  }
}

// A thread has four features of a row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void softmax_join_kernel(SoftmaxArgs A) {
  constexpr int LR = D / 4, RW = kThreads / LR;  // threads of a row, rows of a workgroup
  const SeqGeom& g = A.g;
  const int per = (A.rows + RW - 1) / RW;
  const int row = (int)(blockIdx.x % per) * RW + (int)threadIdx.x / LR, s = blockIdx.x / per, hk = blockIdx.y, f = ((int)threadIdx.x % LR) * 4;
  SeqView v;
  if (!load_seq(g, s, v) || !split_seq(g, v) || row >= v.n * g.G) return;
  const int pieces = (v.L + A.piece - 1) / A.piece;
  if (pieces <= 1) return;
  const long long at = ((long long)s * g.Hkv + hk) * A.splits * A.rows + row;
  float most = -kInf, l = 0.f;
#pragma unroll 8
  for (int k = 0; k < pieces; ++k) most = fmaxf(most, A.sums[at + (long long)k * A.rows].x);
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = 0; k < pieces; ++k) {
    const float2 x = A.sums[at + (long long)k * A.rows];
    const f32x4_t y = *reinterpret_cast<const f32x4_t*>(A.part + (at + (long long)k * A.rows) * D + f);
    const float w = x.y > 0.f ? __builtin_amdgcn_exp2f(x.x - most) : 0.f;
    l = fmaf(x.y, w, l);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], w, o[e]);
  }
  const int t = row / g.G, qh = hk * g.G + row - t * g.G;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T* dst = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + t) * g.o_st + (long long)qh * g.o_sh + f;
  store4<T>(dst, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (f == 0 && A.lse) A.lse[(long long)qh * g.T + v.row0 + t] = l > 0.f ? (most + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
}

template <typename T, int D>
struct SoftmaxTiledCfg {
  static constexpr int KT = sizeof(T) == 4 && D == 128 ? 32 : 64;
  static constexpr int kTileBytes = KT * D * (int)sizeof(T);
  static constexpr size_t kLdsBytes = 4 * (size_t)kTileBytes;
  static constexpr int kWavesPerSimd = sizeof(T) == 4 && D == 128 ? 1 : 2;
};

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(kThreads, (SoftmaxTiledCfg<T, D>::kWavesPerSimd)) void softmax_tiled_kernel(SoftmaxArgs A) {
  using Cfg = SoftmaxTiledCfg<T, D>;
  constexpr int KT = Cfg::KT, NC = D / 16, NM = D / 32, TB = Cfg::kTileBytes;
  using KTile = SeqTile<T, D, KT, false>;
  using Vals = SeqValues<T, D, KT>;
  using VTile = typename Vals::VT;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const SeqGeom& g = A.g;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // (heads and groups in the order of the entmax attention's tiled kernel)
  const int hk = blockIdx.x % g.Hkv, blk = A.nblk - 1 - (int)blockIdx.x / g.Hkv;
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
  const int ntiles = __builtin_amdgcn_readfirstlane((block_lim + KT - 1) / KT);
  const bool holes = seq_has_holes(keys, block_lim);
  const int lane = q.lane;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  FragOff<T> koff[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc) koff[cc] = FragOff<T>::template make<typename KTile::Tile>(q.li, 2 * cc + q.hh);
  Vals vv;
  vv.init(lane);
  typename KTile::Pages pk;
  typename VTile::Pages pv;
  auto ask = [&](int t) {
    pk.ask(keys, t * KT, v.L, wave);
    pv.ask(vals, t * KT, v.L, wave);
  };
  auto issue = [&](int t, int buf) {
    KTile::load(keys, pk, t * KT, v.L, lds0 + (uint32_t)(2 * buf) * TB, wave, lane);
    VTile::load(vals, pv, t * KT, v.L, lds0 + (uint32_t)(2 * buf + 1) * TB, wave, lane);
  };
  if (ntiles > 0) {
    ask(0);
    issue(0, 0);
  }
  if (ntiles > 1) ask(1);
  lds_loads_wait<0>();
  __syncthreads();
  for (int t = 0; t < ntiles; ++t) {
    const int cur = t & 1;
    if (t + 1 < ntiles) {
      issue(t + 1, cur ^ 1);
      if (t + 2 < ntiles) ask(t + 2);
    }
    const char* tile = smem + cur * 2 * TB;
#pragma unroll 1
    for (int sb = 0; sb < KT / 32; ++sb) {
      const int j0 = t * KT + sb * 32;
      if (j0 >= q.lim_max) break;
      const char* at = tile + sb * 32 * KTile::kRowBytes;
      f32x16_t acc = q.scores(q.start(j0), [&](int cc) { return koff[cc].load(at, 0); });
      if constexpr (CAP) q.cap_scores(acc, j0);
      const bool masked = holes || j0 + 32 > q.lim_min;
      if (masked) q.mask(acc, j0, keys, holes);
      float p[16];
      q.step(acc, p);
      vv.accumulate(tile + TB, sb, p, masked, q.oacc);
    }
    lds_loads_wait<0>();
    __syncthreads();
  }
  const float l = q.sum + __shfl_xor(q.sum, 32);
  if (!q.valid) return;
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

// Enqueues the call for checked parameters; returns an entmax_attn_status.
template <typename T, int D>
int run_softmax(const SoftmaxCall& c);

namespace {

// NQB: blocks of 32 rows of a workgroup
template <typename T, int D, int NQB, bool CAP>
bool launch_softmax_split(const SoftmaxArgs& a, hipStream_t st) {
  using Cfg = SoftmaxSplitCfg<T, D>;
  constexpr auto kern = softmax_split_kernel<T, D, NQB, CAP>;
  if (!ensure_dynamic_lds<kern>(Cfg::kLdsBytes)) return false;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.g.nseq * a.splits), (unsigned)a.g.Hkv, (unsigned)ceil_div(a.rows, NQB * 32)), dim3(Cfg::NW * 64), Cfg::kLdsBytes, st, a);
  return launch_ok();
}

template <typename T, int D, bool CAP>
bool launch_softmax(const SoftmaxArgs& a, const SoftmaxLayout& L, hipStream_t st) {
  if (L.blocks) {
    using Cfg = SoftmaxTiledCfg<T, D>;
    constexpr auto kern = softmax_tiled_kernel<T, D, CAP>;
    if (!ensure_dynamic_lds<kern>(Cfg::kLdsBytes)) return false;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.nblk * a.g.Hkv)), dim3(kThreads), Cfg::kLdsBytes, st, a);
    if (!launch_ok()) return false;
  }
  if (!L.split) return true;
  // (two blocks of fp32 rows of 128 features do not fit the registers)
  constexpr int kMostBlocks = sizeof(T) == 4 && D == 128 ? 1 : 2;
  if (!(a.rows <= 32 ? launch_softmax_split<T, D, 1, CAP>(a, st) : launch_softmax_split<T, D, kMostBlocks, CAP>(a, st))) return false;
  if (a.splits > 1) {
    constexpr int RW = kThreads / (D / 4);
    hipLaunchKernelGGL((softmax_join_kernel<T, D>), dim3((unsigned)(a.g.nseq * ceil_div(a.rows, RW)), (unsigned)a.g.Hkv), dim3(kThreads), 0, st, a);
    return launch_ok();
  }
  return true;
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
  a.rows = L.rows;
  a.piece = L.piece;
  a.splits = L.splits;
  a.nblk = (int)seq_blocks(p->nseq, p->T, a.g.G);
  a.split = L.split ? 1 : 0;
  const bool ok = c.cap > 0.f ? launch_softmax<T, D, true>(a, L, c.st) : launch_softmax<T, D, false>(a, L, c.st);
  return ok ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // namespace entmax
