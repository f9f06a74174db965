// Serving attention of sequences with few new tokens (at most kSplitRows folded rows of a key/value head) against any number of keys: the keys, not
// the rows, are split over the chip, and the bound is reading K once.
//   seq_scores_kernel  raw scores d of the rows (y = (alpha-1) s = a d) for a piece of the keys, on the matrix cores straight from
//                      memory, to the workspace, with the largest of every row and block of 32 keys.  A row's scores of a block are
//                      written only if y of the largest is at least that of the largest so far less one: the others have no term at the
//                      lowest possible threshold.  (So whoever knows a row's largest score knows from a block's whether it was written.)
//   seq_solve_kernel   a workgroup per row: candidates, threshold, and, where they are few, the output from the values of the support
//   seq_pv_kernel      rows with long supports: O^T = V^T P^T from the scores, keys split again; the last workgroup of a head adds the parts up
// Measured, bf16: 64 x 1 token, 2 x 8 heads of 128, 200 to 8192 keys: 21 + 11 + 4 us (K 62 MB: 3 TB/s, the lengths end at different times); 4 x 1 token,
// 4 x 3 heads of 64, 32768 keys: 16 + 8 + 3 us (K at 4.2 TB/s).  Rows that keep most of 8192 to 16384 keys, 8 x 1 token, 4 x 4 heads of 128: 24 + 30 + 34 us,
// bound by the solve's passes over whole rows of scores, and by V and the scores a second time.
// From the second kernel on y and the threshold are taken relative to the row's largest score (y = a (d - top), tau in [-1, 0)): large scores then cost no
// bits of the probabilities.
#pragma once
#include "decode.hip.h"
#include "seq.hip.h"
#include "seq_layout.h"
#include "seq_tiled.hip.h"

namespace entmax {

struct SeqDecodeArgs {
  SeqGeom g;
  const void* Q;
  const void* K;
  const void* V;
  void* O;
  float* scores;     // [nseq * Hkv][rows][32 nblk]
  float* bmax;       // [nseq * Hkv][rows][nblk] largest score of each 32-key block that starts before the sequence's end
  float* mult;       // [nseq * Hkv][rows] the rows' a
  float2* found;     // [nseq * Hkv][rows] (threshold, or +inf: the row is finished; largest score)
  int* arrived;      // [nseq * Hkv] workgroups of seq_pv_kernel that have left their part
  float* part;       // [nseq * Hkv][pv_splits][rows][D]
  int rows;          // rows of a head there is room for: min(max_new G, kSplitRows)
  int nblk;          // 32-key blocks of max_keys
  int run, splits;           // seq_scores_kernel: consecutive blocks of a wave, workgroups of a head
  int pv_keys, pv_splits;    // seq_pv_kernel: keys of a workgroup, workgroups of a head
};

// How far below the row's largest raw score a key may lie and still have a term at the lowest threshold (a little more, for the rounding)
__device__ __forceinline__ float score_reach(float a) { return 1.00001f / a; }

template <typename T, int D, int NQB>
__global__ __launch_bounds__(kThreads) void seq_scores_kernel(SeqDecodeArgs A) {
  constexpr int NC = D / 16;
  __shared__ int rowmax[NQB * 32];  // ordered_bits() of a row's largest score so far
  const SeqGeom& g = A.g;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, li = lane & 31, hh = lane >> 5;
  const int split = blockIdx.x % A.splits, s = blockIdx.x / A.splits, hk = blockIdx.y;
  const int head = s * g.Hkv + hk;
  if (split == 0 && tid == 0) A.arrived[head] = 0;
  SeqView v;
  if (!load_seq(g, s, v) || !split_seq(g, v)) return;
  if (split * kWaves * A.run * 32 >= v.L) return;
  const int blk0 = (split * kWaves + wave) * A.run, end = min(blk0 + A.run, (v.L + 31) >> 5);  // this wave's blocks (there may be none)
  SeqKeys keys;
  keys.init(g, v, A.K, hk, false, sizeof(T));
  auto page_of = [&](int blk) { return keys.page(min(blk * 32 + li, v.L - 1)); };
  Frag<T> kf[NC], kn[NC];
  auto fetch = [&](Frag<T>* dst, int blk, int pg) {  // (rows past the end repeat the last one; their scores are masked)
    const char* row = keys.row_in(pg, min(blk * 32 + li, v.L - 1)) + 8 * hh * sizeof(T);
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) dst[cc] = Elem<T>::load(row + 16 * cc * sizeof(T));
  };
  int pg = 0, pg_next = 0;  // pages of the block in kn and of the one after it
  if (blk0 < end) {
    pg = page_of(blk0);
    pg_next = page_of(min(blk0 + 1, end - 1));
    fetch(kn, blk0, pg);
  }
  const int R = v.n * g.G;
  SeqRows<T, D> q[NQB];
  float top[NQB], reach[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    q[qb].init(g, v, A.Q, hk, qb * 32);
    top[qb] = -kInf;
    reach[qb] = score_reach(q[qb].a);
    if (split == 0 && wave == 0 && hh == 0 && q[qb].valid) A.mult[(long long)head * A.rows + qb * 32 + li] = q[qb].a;
  }
  if (tid < NQB * 32) rowmax[tid] = ordered_bits(-kInf);
  __syncthreads();
  for (int blk = blk0; blk < end; ++blk) {
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) kf[cc] = kn[cc];
    const uint32_t holes = (uint32_t)__ballot(keys.is_hole(pg));  // of the block's 32 keys
    if (blk + 1 < end) {
      pg = pg_next;
      pg_next = page_of(min(blk + 2, end - 1));
      fetch(kn, blk + 1, pg);
    }
    const int j0 = blk * 32;
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      if (qb * 32 >= R) break;
      f32x16_t acc = q[qb].dots(q[qb].start(j0), [&](int cc) { return kf[cc]; });
      if (j0 + 32 > q[qb].lim_min || holes != 0u) {
        const int rel = q[qb].lim - j0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int k = q[qb].key_of(e);
          acc[e] = k < rel && ((holes >> k) & 1u) == 0u ? acc[e] : -kInf;
        }
      }
      float m = max16(acc);
      m = fmaxf(m, __shfl_xor(m, 32));
      const long long row = (long long)head * A.rows + qb * 32 + li;
      if (hh == 0 && q[qb].valid) A.bmax[row * A.nblk + blk] = m;
      // (an older value only writes more)
      top[qb] = fmaxf(top[qb], from_ordered_bits(__hip_atomic_load(&rowmax[qb * 32 + li], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)));
      // (m = -inf for rows that see none of the block; the row's first lane decides for both)
      const uint32_t rows = (uint32_t)__ballot(m > -kInf && m >= top[qb] - reach[qb] && q[qb].lim > 0);
      if ((rows >> li) & 1u) {
        if (m > top[qb]) {
          top[qb] = m;
          atomicMax(&rowmax[qb * 32 + li], ordered_bits(m));
        }
        float* dst = A.scores + (row * A.nblk + blk) * 32 + 4 * hh;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<f32x4_t*>(dst + 8 * q4) = f32x4_t{acc[4 * q4], acc[4 * q4 + 1], acc[4 * q4 + 2], acc[4 * q4 + 3]};
      }
    }
  }
}

// Sums over the workgroup (NT threads) of three values and the smallest of a fourth, the same in every thread.  Calls alternate between
// the halves of buf (parity), so that one barrier per call is enough.
template <int NT>
__device__ __forceinline__ RowSums block_sums(RowSums s, float* buf, int parity) {
  constexpr int kW = NT / 64;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    s.s0 += __shfl_xor(s.s0, off);
    s.s1 += __shfl_xor(s.s1, off);
    s.s2 += __shfl_xor(s.s2, off);
    s.xmin = fminf(s.xmin, __shfl_xor(s.xmin, off));
  }
  f32x4_t* mine = reinterpret_cast<f32x4_t*>(buf) + parity * kW;
  if ((threadIdx.x & 63) == 0) mine[threadIdx.x >> 6] = f32x4_t{s.s0, s.s1, s.s2, s.xmin};
  __syncthreads();
  RowSums t;
  t.clear();
#pragma unroll
  for (int w = 0; w < kW; ++w) {
    const f32x4_t o = mine[w];
    t.s0 += o[0];
    t.s1 += o[1];
    t.s2 += o[2];
    t.xmin = fminf(t.xmin, o[3]);
  }
  return t;
}

constexpr int kSolveList = 256;   // candidates kept in LDS, their output gathered here; rows with more are left to seq_pv_kernel
// Rows with more 32-key blocks than this within reach get a higher floor from the blocks' largest scores first.  8 tokens x 16 heads of 128 against
// 32000 keys, logits without a scale: 19 us, and 4 us for the values; without the floor 73 us, and 54 us.  Rows of few such blocks are spared its
// passes (no difference seen at 1 to 5 tokens against up to 32768 keys with scales).
constexpr int kSolveManyBlocks = 24;
constexpr int kSolveHeld = 16;    // scores of a long row that a thread holds in registers

template <typename T, int D, int NT>
struct SolveLds {
  static constexpr int kW = NT / 64;
  float2 list[kSolveList];  // (key index bits, raw score, then y)
  __attribute__((aligned(16))) float red[2 * kW * 4];
  float wtop[kW];
  int whot[kW];
  int count;
  float osum[kW * D];
};

template <typename T, int D, int AM, int NT>
__device__ __forceinline__ void solve_row(const SeqDecodeArgs& A, SolveLds<T, D, NT>& lds, const SeqView& v, int head, int row) {
  constexpr int kW = NT / 64;
  constexpr int E = 16 / (int)sizeof(T), LR = D / E;  // features of a lane, lanes of a value row
  constexpr int kGroups = NT / LR;
  float2* list = lds.list;
  float *red = lds.red, *wtop = lds.wtop, *osum = lds.osum;
  int& count = lds.count;
  const SeqGeom& g = A.g;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hk = head % g.Hkv, t = row / g.G, qh = hk * g.G + row % g.G;
  const int lim = g.causal ? max(0, min(v.L - v.n + t + 1, v.L)) : v.L;
  const long long at = (long long)head * A.rows + row;
  T* o = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + t) * g.o_st + (long long)qh * g.o_sh;
  const float* d = A.scores + at * A.nblk * 32;
  const float* bmax = A.bmax + at * A.nblk;
  const int nblk = (v.L + 31) >> 5;
  const float a = A.mult[at], reach = score_reach(a);
  const float r = 1.0f / (g.alpha - 1.0f);
  SeqKeys vals;
  vals.init(g, v, A.V, hk, true, sizeof(T));
  // the largest score from the blocks' (the first NT of them are held)
  const float first = tid < nblk ? bmax[tid] : -kInf;
  float top = first;
  for (int b = tid + NT; b < nblk; b += NT) top = fmaxf(top, bmax[b]);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  if (lane == 0) wtop[wave] = top;
  if (tid == 0) count = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kW; ++w) top = fmaxf(top, wtop[w]);
  if (lim == 0 || top == -kInf) {  // no visible key: an empty sum
    if (tid < D) Elem<T>::store(o, tid, 0.f);
    if (tid == 0) A.found[at] = make_float2(kInf, 0.f);
    return;
  }
  float floor_lo = top - reach;  // (at most top, which is always a candidate)
  auto hot = [&](float m) { return m >= floor_lo && m > -kInf; };
  // y = a (d - top) in [-1, 0]: the threshold lies between -1 and -n^(1-alpha)
  auto y_of = [&](float x) { return a * (x - top); };
  float lo = -1.0f, hi = -__builtin_amdgcn_exp2f(-(g.alpha - 1.0f) * __builtin_amdgcn_logf((float)lim));
  {
    // Where many blocks come within reach: Newton steps from the left on the blocks' largest scores (scores of different keys: dropping the others
    // can only lower the threshold) give a higher floor, and far fewer candidates.
    const unsigned long long mine = __ballot(hot(first));
    if (lane == 0) lds.whot[wave] = (int)__popcll(mine);
    __syncthreads();
    int blocks = 0;
#pragma unroll
    for (int w = 0; w < kW; ++w) blocks += lds.whot[w];
    if (blocks > kSolveManyBlocks) {
      float t = -1.0f;
      for (int it = 0; it < 4; ++it) {
        RowSums sums;
        sums.clear();
        auto term = [&](float m) {
          const float x = hot(m) ? fmaxf(y_of(m) - t, 0.f) : 0.f;
          const float gx = x > 0.f ? pow_rm1<AM>(x, r) : 0.f;
          sums.s0 += gx;
          sums.s1 = fmaf(gx, x, sums.s1);
        };
        term(first);
        for (int b = tid + NT; b < nblk; b += NT) term(bmax[b]);
        sums = block_sums<NT>(sums, red, it & 1);
        if (!(sums.s1 > 1.0f)) break;  // (the same in every thread)
        t += (sums.s1 - 1.0f) / (r * sums.s0);
      }
      lo = fminf(fmaxf(lo, t - 4e-6f), hi);
      floor_lo = fmaf(lo, reach, top);
      __syncthreads();  // (red is used again)
    }
  }
  float tau = lo;
  // the candidates: two blocks of a wave at a time, half a wave each, and two such pairs under way; a row with more than the list holds is
  // counted no further
  for (int b0 = 0; b0 < nblk; b0 += NT) {
    const int b = b0 + tid;
    const float m = b0 == 0 ? first : (b < nblk ? bmax[b] : -kInf);
    unsigned long long todo = __ballot(b < nblk && hot(m));
    while (todo != 0ull) {
      if (__hip_atomic_load(&count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > kSolveList) break;
      int mine[2];
      float x[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int k0 = todo != 0ull ? __builtin_ctzll(todo) : -1;
        todo &= todo - 1ull;  // (0 stays 0)
        const int k1 = todo != 0ull ? __builtin_ctzll(todo) : -1;
        todo &= todo - 1ull;
        mine[u] = lane < 32 ? k0 : k1;
        x[u] = mine[u] >= 0 ? d[(b0 + wave * 64 + mine[u]) * 32 + (lane & 31)] : -kInf;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bool in = hot(x[u]);
        const unsigned long long all = __ballot(in);
        if (all == 0ull) continue;
        int pos = 0;
        if (lane == 0) pos = atomicAdd(&count, (int)__popcll(all));
        pos = __builtin_amdgcn_readfirstlane(pos) +
              (int)__builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, 0u));
        if (in && pos < kSolveList) list[pos] = make_float2(__int_as_float((b0 + wave * 64 + mine[u]) * 32 + (lane & 31)), x[u]);
      }
    }
  }
  __syncthreads();
  const int total = count;
  // features of this lane of the value row of key j, times p
  auto add_row = [&](int j, float p, float (&acc)[E]) {
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(vals.row(j) + (lane % LR) * 16);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(p, word_elem<T>(w, e), acc[e]);
  };
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;

  // The candidates come in the order in which the waves found them; the sums go in the order of the keys.
  auto rank_of = [&](int key) {
    int rank = 0;
    for (int k = 0; k < total; ++k) rank += __float_as_int(list[k].x) < key ? 1 : 0;
    return rank;
  };
  if (total <= 64) {  // one wave's, in registers
    if (wave != 0) return;
    float2 en = make_float2(0.f, 0.f);
    if (lane < total) en = list[lane];
    const int rank = rank_of(__float_as_int(en.x));
    __builtin_amdgcn_wave_barrier();
    if (lane < total) list[rank] = en;
    __builtin_amdgcn_wave_barrier();
    if (lane < total) en = list[lane];
    const float y = lane < total ? y_of(en.y) : -kInf;
    bool done = false;
    for (int it = 0; !done && it < kMaxSolveIters; ++it) {
      RowSums sums;
      sums.clear();
      accumulate<AM>(sums, y - tau, r);
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) {
        sums.s0 += __shfl_xor(sums.s0, off);
        sums.s1 += __shfl_xor(sums.s1, off);
        sums.s2 += __shfl_xor(sums.s2, off);
        sums.xmin = fminf(sums.xmin, __shfl_xor(sums.xmin, off));
      }
      done = solve_step<AM>(sums, r, tau, lo, hi);
    }
    const float p = lane < total ? pow_r<AM>(fmaxf(y - tau, 0.f), r) : 0.f;
    unsigned long long sup = __ballot(p > 0.f);
    const int grp = lane / LR;
    constexpr int WG = 64 / LR;  // value rows of the wave at a time
    while (sup != 0ull) {
      int mine = -1;
#pragma unroll
      for (int u = 0; u < WG; ++u) {
        const int k = sup != 0ull ? __builtin_ctzll(sup) : -1;
        sup &= sup - 1ull;  // (0 stays 0)
        if (u == grp) mine = k;
      }
      const float pk = __shfl(p, max(mine, 0));
      const int j = __shfl(__float_as_int(en.x), max(mine, 0));
      if (mine >= 0) add_row(j, pk, acc);
    }
#pragma unroll
    for (int off = LR; off < 64; off <<= 1)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += __shfl_xor(acc[e], off);
    if (lane < LR) {
#pragma unroll
      for (int e = 0; e < E; e += 4) store4<T>(o + lane * E + e, acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    }
    if (lane == 0) A.found[at] = make_float2(kInf, 0.f);
    return;
  }
  // tau from n values y_at(e)
  auto solve = [&](auto y_at, int n) {
    bool done = false;
    for (int it = 0; !done && it < kMaxSolveIters; ++it) {
      RowSums sums;
      sums.clear();
      for (int e = tid; e < n; e += NT) accumulate<AM>(sums, y_at(e) - tau, r);
      sums = block_sums<NT>(sums, red, it & 1);
      done = solve_step<AM>(sums, r, tau, lo, hi);
    }
  };
  if (total <= kSolveList) {
    static_assert(kSolveList <= NT, "a thread per candidate");
    float2 en = make_float2(0.f, 0.f);
    int rank = 0;
    if (tid < total) {
      en = list[tid];
      rank = rank_of(__float_as_int(en.x));
    }
    __syncthreads();
    if (tid < total) list[rank] = make_float2(en.x, y_of(en.y));
    __syncthreads();
    solve([&](int e) { return list[e].y; }, total);
    for (int e = tid / LR; e < total; e += kGroups) {
      const float x = list[e].y - tau;
      if (x > 0.f) add_row(__float_as_int(list[e].x), pow_r<AM>(x, r), acc);
    }
    // lanes of equal features: within the wave, then over the waves in their order
#pragma unroll
    for (int off = LR; off < 64; off <<= 1)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += __shfl_xor(acc[e], off);
    if (lane < LR) {
#pragma unroll
      for (int e = 0; e < E; ++e) osum[wave * D + lane * E + e] = acc[e];
    }
    __syncthreads();
    if (tid < D) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kW; ++w) sum += osum[w * D + tid];
      Elem<T>::store(o, tid, sum);
    }
    if (tid == 0) A.found[at] = make_float2(kInf, 0.f);
    return;
  }
  // Long supports.  Key e of the row counts if its block was written; -inf (y far below -1) else.  The first kSolveHeld NT of them are read once.
  const int n = nblk * 32;
  auto y_at = [&](int e) {
    const float m = bmax[min(e, n - 1) >> 5], x = d[min(e, n - 1)];  // (two loads, not one after the other)
    return e < n && hot(m) ? y_of(x) : -kInf;
  };
  float held[kSolveHeld];
#pragma unroll
  for (int k = 0; k < kSolveHeld; ++k) held[k] = y_at(tid + k * NT);
  auto each = [&](auto fn) {
#pragma unroll
    for (int k = 0; k < kSolveHeld; ++k) fn(held[k]);
    for (int e = tid + kSolveHeld * NT; e < n; e += 4 * NT) {
      float y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = y_at(e + u * NT);
#pragma unroll
      for (int u = 0; u < 4; ++u) fn(y[u]);
    }
  };
  bool done = false;
  for (int it = 0; !done && it < kMaxSolveIters; ++it) {
    RowSums sums;
    sums.clear();
    each([&](float y) { accumulate<AM>(sums, y - tau, r); });
    sums = block_sums<NT>(sums, red, it & 1);
    done = solve_step<AM>(sums, r, tau, lo, hi);
  }
  if (tid == 0) A.found[at] = make_float2(tau, top);
}

// NT: threads of a workgroup.  It takes the rows blockIdx.x % stride, + stride, .. of a head (one, but where few sequences of many have many rows).
template <typename T, int D, int AM, int NT>
__global__ __launch_bounds__(NT) void seq_solve_kernel(SeqDecodeArgs A, int stride) {
  __shared__ SolveLds<T, D, NT> lds;
  const int head = blockIdx.x / stride, s = head / A.g.Hkv;
  SeqView v;
  if (!load_seq(A.g, s, v) || !split_seq(A.g, v)) return;
  for (int row = blockIdx.x % stride; row < v.n * A.g.G; row += stride) {
    solve_row<T, D, AM, NT>(A, lds, v, head, row);
    __syncthreads();
  }
}

// Keys of a wave's tile of V and its bytes: one tile per wave in LDS, the next one waits in registers
template <typename T, int D>
struct SeqPvCfg {
  static constexpr int KT = 32;
  static constexpr int kTileBytes = KT * D * (int)sizeof(T);
};

// four floats to and from memory at agent scope
__device__ __forceinline__ void put_part(float* at, const f32x4_t& x) {
  unsigned long long* p = reinterpret_cast<unsigned long long*>(at);
#pragma unroll
  for (int k = 0; k < 2; ++k)
    __hip_atomic_store(p + k, (unsigned long long)__float_as_uint(x[2 * k]) | (unsigned long long)__float_as_uint(x[2 * k + 1]) << 32, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4_t get_part(const float* at) {
  const unsigned long long* p = reinterpret_cast<const unsigned long long*>(at);
  f32x4_t x;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const unsigned long long v = __hip_atomic_load(p + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    x[2 * k] = __uint_as_float((uint32_t)v);
    x[2 * k + 1] = __uint_as_float((uint32_t)(v >> 32));
  }
  return x;
}

// O^T = V^T P^T for the rows that seq_solve_kernel left (tau finite).  Every wave goes through its own 32-key blocks of the workgroup's
// piece of the keys; the waves' sums are added in their order, and the workgroup that comes last adds up the pieces in theirs.
template <typename T, int D, int AM, int NQB>
__global__ __launch_bounds__(kThreads) void seq_pv_kernel(SeqDecodeArgs A) {
  constexpr int NM = D / 32, KT = SeqPvCfg<T, D>::KT;
  using Vals = SeqValues<T, D, KT>;
  __shared__ __attribute__((aligned(16))) char tiles[kWaves * SeqPvCfg<T, D>::kTileBytes];
  __shared__ int last;
  const SeqGeom& g = A.g;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, li = lane & 31, hh = lane >> 5;
  const int split = blockIdx.x % A.pv_splits, s = blockIdx.x / A.pv_splits, hk = blockIdx.y;
  const int head = s * g.Hkv + hk;
  SeqView v;
  if (!load_seq(g, s, v) || !split_seq(g, v)) return;
  const int from = split * A.pv_keys;
  if (from >= v.L) return;
  const int R = v.n * g.G;
  float tau[NQB], top[NQB], a[NQB];
  bool left[NQB];
  bool any = false;
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int row = qb * 32 + li;
    const long long at = (long long)head * A.rows + row;
    const float2 f = row < R ? A.found[at] : make_float2(kInf, 0.f);
    a[qb] = row < R ? A.mult[at] : 1.f;
    tau[qb] = f.x;
    top[qb] = f.y;
    left[qb] = tau[qb] < kInf;
    any = any || left[qb];
  }
  if (__ballot(any) == 0ull) return;  // (the same for all waves)
  const int to = min(v.L, from + A.pv_keys), nblk = (to - from + 31) >> 5;
  const float r = 1.0f / (g.alpha - 1.0f);
  SeqKeys vals;
  vals.init(g, v, A.V, hk, true, sizeof(T));
  // keys from this one on are not seen by every row; with holes, none is (SeqValues::accumulate())
  int all_see = g.causal ? max(0, v.L - v.n + 1) : v.L;
  {
    int bad = 0;
    for (int e = (from >> g.lps) + tid; e << g.lps < to; e += kThreads) bad |= vals.is_hole(vals.page(e << g.lps)) ? 1 : 0;
    if (__syncthreads_or(bad)) all_see = 0;
  }
  char* tile = tiles + wave * SeqPvCfg<T, D>::kTileBytes;
  Vals vv;
  vv.init(lane);
  f32x16_t oacc[NQB][NM];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
    for (int mm = 0; mm < NM; ++mm)
      oacc[qb][mm] = f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // the wave's tile: 64 lanes bring 1024 bytes at a time
  using VT = typename Vals::VT;
  constexpr int CPR = VT::kCpr, RW = VT::RW, L = KT / RW;
  u32x4_t stage[L];
  f32x4_t ys[NQB][4];
  int pages[L];       // of the block after the one that is fetched next
  float best[NQB];    // its largest score of this lane's row
  auto ask = [&](int blk) {
    const int j0 = from + min(blk, nblk - 1) * 32;
#pragma unroll
    for (int it = 0; it < L; ++it) pages[it] = vals.page(min(j0 + it * RW + lane / CPR, v.L - 1));
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
      best[qb] = left[qb] ? A.bmax[((long long)head * A.rows + qb * 32 + li) * A.nblk + (j0 >> 5)] : -kInf;
  };
  auto fetch = [&](int blk) {
    const int j0 = from + blk * 32;
#pragma unroll
    for (int it = 0; it < L; ++it)
      stage[it] = *reinterpret_cast<const u32x4_t*>(vals.row_in(pages[it], min(j0 + it * RW + lane / CPR, v.L - 1)) + (lane % CPR) * 16);
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      if (qb * 32 >= R) break;
      // (what was not written has no term)
      const bool there = best[qb] > -kInf && best[qb] >= top[qb] - score_reach(a[qb]);
      const float* y = A.scores + (((long long)head * A.rows + qb * 32 + li) * A.nblk + (j0 >> 5)) * 32 + 4 * hh;
#pragma unroll
      for (int k = 0; k < 4; ++k) ys[qb][k] = there ? *reinterpret_cast<const f32x4_t*>(y + 8 * k) : f32x4_t{-kInf, -kInf, -kInf, -kInf};
    }
  };
  if (wave < nblk) {
    ask(wave);
    fetch(wave);
    ask(wave + kWaves);
  }
  for (int blk = wave; blk < nblk; blk += kWaves) {
    __builtin_amdgcn_wave_barrier();  // (the tile is the wave's own: LDS operations of a wave are in order)
#pragma unroll
    for (int it = 0; it < L; ++it) {
      const int row = it * RW + lane / CPR;
      *reinterpret_cast<u32x4_t*>(tile + VT::off(row, lane % CPR)) = stage[it];
    }
    float p[NQB][16];
    const int j0 = from + blk * 32;
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      if (qb * 32 >= R) break;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = fmaf(a[qb], ys[qb][e >> 2][e & 3] - top[qb], -tau[qb]);
        p[qb][e] = left[qb] ? pow_r<AM>(fmaxf(x, 0.f), r) : 0.f;
      }
    }
    if (blk + kWaves < nblk) {
      fetch(blk + kWaves);
      ask(blk + 2 * kWaves);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      if (qb * 32 >= R) break;
      bool some = false;
#pragma unroll
      for (int e = 0; e < 16; ++e) some = some || p[qb][e] > 0.f;
      if (__ballot(some) != 0ull) vv.accumulate(tile, 0, p[qb], j0 + 32 > all_see, oacc[qb]);
    }
  }
  // the waves' sums in LDS, 32 rows and one 32-feature block at a time: [wave][16][64]
  float* red = reinterpret_cast<float*>(tiles);
  static_assert(SeqPvCfg<T, D>::kTileBytes >= 16 * 64 * 4, "a wave's accumulators fit its tile");
  float* part = A.part + ((long long)head * A.pv_splits + split) * A.rows * D;
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    if (qb * 32 >= R) break;
#pragma unroll
    for (int mm = 0; mm < NM; ++mm) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 16; ++e) red[(wave * 16 + e) * 64 + lane] = oacc[qb][mm][e];
      __syncthreads();
      // thread: row tid % 32 (of half tid / 32 % 2), accumulators 4 (tid / 64) .. + 3
      f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += red[(w * 16 + 4 * wave + e) * 64 + lane];
      const int row = qb * 32 + li;
      if (row < R) put_part(part + (long long)row * D + 32 * mm + 8 * wave + 4 * hh, sum);
    }
  }
  // The parts pass through memory that all XCDs see: written and read by operations of agent scope, each workgroup's finished (the wait of
  // every wave, then the barrier) before it counts itself.  A fence of agent scope would write back the whole L2, for every workgroup
  // (decode_dense, 768 of them: 118 us).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const int parts = (v.L + A.pv_keys - 1) / A.pv_keys;
  if (tid == 0) last = __hip_atomic_fetch_add(&A.arrived[head], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1 ? 1 : 0;
  __syncthreads();
  if (last == 0) return;
  const float* all = A.part + (long long)head * A.pv_splits * A.rows * D;
  for (int e = tid; e < R * (D / 4); e += kThreads) {
    const int row = e / (D / 4), f = (e % (D / 4)) * 4;
    if (!(A.found[(long long)head * A.rows + row].x < kInf)) continue;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int k = 0; k < parts; ++k) {
      const f32x4_t x = get_part(all + ((long long)k * A.rows + row) * D + f);
#pragma unroll
      for (int u = 0; u < 4; ++u) sum[u] += x[u];
    }
    T* o = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + row / g.G) * g.o_st + (long long)(hk * g.G + row % g.G) * g.o_sh + f;
    store4<T>(o, sum[0], sum[1], sum[2], sum[3]);
  }
}

}  // namespace entmax
