// Sequences of different lengths with grouped heads over packed or paged keys: what the serving kernels share.
//   SeqGeom   the problem, as the entry points hand it to the kernels
//   SeqView   one sequence: its rows of Q and O, its keys (load_seq checks what the device arrays say)
//   SeqKeys   addresses of a sequence's key (or value) rows, by page or packed
//   SeqRows   a wave's 32 folded rows.  The rows of a key/value head are (token, query head of the group) with the head
//             running fastest: 32 consecutive ones share every key, so that one read of a key serves the whole group.
#pragma once
#include "qside.hip.h"

namespace entmax {

struct SeqGeom {
  int nseq, T, Hq, Hkv, G;  // G = Hq / Hkv
  int causal, scale_layout, logn_mode, bias_mode;
  float alpha, delta;
  const float* beta;
  const float* gamma;
  const float* slopes;
  const int* cu;       // [nseq + 1]
  const int* kv_len;   // [nseq]; NULL: packed, as many keys as tokens
  const int* table;    // [nseq][max_pages]; NULL: packed
  int lps;             // log2 of the page size (packed: 4, "pages" of 16 consecutive rows)
  int num_pages, max_pages, max_new, max_keys;
  long long q_st, q_sh, o_st, o_sh;      // element strides
  long long k_sp, k_sh, k_sn, v_sp, v_sh, v_sn;
};

struct SeqView {
  int s, row0, n, L;  // sequence, its first row of Q, new tokens, keys
};

// What the arrays say of sequence s; false: it is left out.  (Values are compared before anything is computed from them.)
__device__ __forceinline__ bool load_seq(const SeqGeom& g, int s, SeqView& v) {
  const int from = g.cu[s], to = g.cu[s + 1];
  v.s = s;
  v.row0 = from;
  if (from < 0 || to > g.T || to <= from) return false;
  v.n = to - from;
  v.L = g.kv_len ? g.kv_len[s] : v.n;
  return v.n <= g.max_new && v.L >= 0 && v.L <= g.max_keys;
}

// Number of entries i in 1 .. nseq with f(cu[i], i) <= x, for f that does not decrease: the sequence that row or block x belongs to (nseq:
// it lies behind the last one).  All 64 lanes of the wave together: 64 entries are compared at a time, of long arrays first every
// 64th, so that the search is one or two memory round trips (nseq <= 4096; one more for each further 64-fold).
template <class F>
__device__ __forceinline__ int find_seq(const int* cu, int nseq, long long x, F f) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = nseq;  // entries 1 .. lo are <= x; the answer is in lo .. lo + n
  while (n > 0) {
    const int step = (n + 63) >> 6;
    const int i = lo + min((lane + 1) * step, n);
    const bool in = lane * step < n;
    const int below = (int)__popcll(__ballot(in && f(cu[in ? i : 0], i) <= x));
    // lanes 0 .. below - 1 hold: their last entry is <= x, and lane `below`'s (if there is one) is not
    const int got = min(below * step, n);
    const int rest = below * step < n ? min(step, n - below * step) - 1 : 0;
    lo += got;
    n = step == 1 ? 0 : rest;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Rows of one key/value head of a sequence, as bytes.
struct SeqKeys {
  // (constant memory for the time of a kernel: numbers for uniform places come through the scalar cache, and waiting for them is not
  // waiting for the tiles under way)
  typedef const __attribute__((address_space(4))) int* Pages;
  const char* base;  // of the head (packed: of the sequence's first row)
  Pages pages;       // the sequence's row of the page table
  bool paged;
  long long sp, sn;  // byte strides of pages and rows
  int lps, num_pages;
  __device__ __forceinline__ void init(const SeqGeom& g, const SeqView& v, const void* X, int hk, bool values, int esize) {
    const long long sn_e = values ? g.v_sn : g.k_sn, sh_e = values ? g.v_sh : g.k_sh, sp_e = values ? g.v_sp : g.k_sp;
    sn = sn_e * esize;
    paged = g.table != nullptr;
    pages = (Pages)(paged ? g.table + (long long)v.s * g.max_pages : g.cu);
    sp = paged ? sp_e * esize : sn << g.lps;
    base = reinterpret_cast<const char*>(X) + hk * sh_e * esize + (paged ? 0 : (long long)v.row0 * sn);
    lps = g.lps;
    num_pages = g.num_pages;
  }
  // page of key j (0 <= j < L); a hole: not in 0 .. num_pages - 1
  // (read in either case, packed from a place that is always there: no branch that the loads would wait for one by one)
  __device__ __forceinline__ int page(int j) const {
    const int x = j >> lps, y = pages[paged ? x : 0];
    return paged ? y : x;
  }
  __device__ __forceinline__ bool is_hole(int pg) const { return paged && (unsigned)pg >= (unsigned)num_pages; }
  // (a hole's keys are masked wherever they are used; they are read from page 0)
  __device__ __forceinline__ const char* row_in(int pg, int j) const {
    return base + (long long)(is_hole(pg) ? 0 : pg) * sp + (long long)(j & ((1 << lps) - 1)) * sn;
  }
  __device__ __forceinline__ const char* row(int j) const { return row_in(page(j), j); }
};

// Whether any page of keys 0 .. L - 1 is a hole; all threads of the workgroup together (a barrier).
__device__ __forceinline__ bool seq_has_holes(const SeqKeys& k, int L) {
  if (!k.paged) return false;  // (uniform)
  int bad = 0;
  for (int e = threadIdx.x; e << k.lps < L; e += blockDim.x) bad |= k.is_hole(k.pages[e]) ? 1 : 0;
  return __syncthreads_or(bad) != 0;
}

// One tile of KT rows to LDS without registers in between (load_to_lds()).  16-byte chunks, swizzled by row: SWZ false: as LdsTile, for
// ds_read_b128 of 32 rows at a time (keys) and for reads along a row; true: for transposed reads (values of 2 bytes), where four
// consecutive rows' 32-byte pieces are read together and pairs of chunks must stay together.
// NT: threads of the workgroup.
template <typename T, int D, int KT, bool TR, int NT = kThreads>
struct SeqTile {
  using Tile = LdsTile<T, KT, D>;
  static constexpr int kCpr = Tile::kCpr, kBytes = Tile::kBytes, kRowBytes = Tile::kRowBytes;
  static constexpr int L = Tile::kChunks / NT;  // loads of a wave
  static constexpr int RS = NT / kCpr;          // rows of the tile per load of all waves
  static constexpr int RW = 64 / kCpr;                // rows of a wave's load: within one page (page sizes are multiples of 16)
  static_assert(16 % RW == 0 && Tile::kChunks % NT == 0, "a load's rows lie in one page");
  static __device__ __forceinline__ int swz(int row) {
    if (!TR) return Tile::swz(row);
    return kCpr == 8 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
  }
  static __device__ __forceinline__ int off(int row, int chunk) { return row * kRowBytes + ((chunk ^ swz(row)) << 4); }
  // The pages of the rows that this wave loads of the tile at j0 (asked for one tile ahead)
  struct Pages {
    int pg[L];
    __device__ __forceinline__ void ask(const SeqKeys& k, int j0, int n, int wave) {
#pragma unroll
      for (int it = 0; it < L; ++it) pg[it] = k.page(max(0, min(j0 + it * RS + wave * RW, n - 1)));
    }
  };
  // rows j0 .. j0 + KT - 1 of a sequence of n rows (n > j0); rows behind the last one repeat it.  lds: LDS address of the tile.
  static __device__ __forceinline__ void load(const SeqKeys& k, const Pages& p, int j0, int n, uint32_t lds, int wave, int lane) {
    const int rl = lane / kCpr;
#pragma unroll
    for (int it = 0; it < L; ++it) {
      const int row = it * RS + wave * RW;  // first row of this wave's load
      const uint32_t chunk = (uint32_t)(((lane % kCpr) ^ swz(row + rl)) << 4);
      const uint32_t dst = lds + (uint32_t)((it * NT + wave * 64) * 16);
      if (j0 + KT <= n) {
        load_to_lds(k.row_in(p.pg[it], j0 + row), (uint32_t)rl * (uint32_t)k.sn + chunk, dst);
      } else {
        const char* src = k.row(min(j0 + row + rl, n - 1)) + chunk;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(src) : "memory", "m0");
      }
    }
  }
};

// What belongs to a folded row.
struct SeqRow {
  int t, head;          // token of the sequence, query head
  bool valid;
  int lim, pos;         // keys j < lim are visible; the row's position
  // as in QCtx: y_ij = a d_ij, d_ij = +-<q_i, k_j> + w max(pos - j, 0).  A row of scale 0 (c = 0) has a = 1 and d_ij = 0, so that masked
  // scores are never multiplied by zero.
  float a, c, w;
  // FAST: (ln n)^gamma from the hardware's logarithm and exponential, a few 1e-7 off: it multiplies the distances of scores from the row's largest, at
  // most 1 where they count (kernels with bf16 results)
  template <bool FAST>
  __device__ __forceinline__ void init(const SeqGeom& g, const SeqView& v, int hk, int r, int D) {
    valid = r < v.n * g.G;
    t = valid ? r / g.G : 0;
    head = hk * g.G + (valid ? r - t * g.G : 0);
    pos = v.L - v.n + t;
    lim = !valid ? 0 : (g.causal ? max(0, min(pos + 1, v.L)) : v.L);
    float scale = g.delta;
    if (g.scale_layout != 0) {
      const long long idx = g.scale_layout == 1 ? head : (long long)head * g.T + v.row0 + t;
      const int n = g.logn_mode == 0 ? v.L : lim;
      const float be = g.beta[idx], ga = g.gamma[idx];
      if (n > 1) {
        const float ln = FAST ? __builtin_amdgcn_logf((float)n) * 0.69314718f : logf((float)n);
        scale += be * (FAST ? __builtin_amdgcn_exp2f(ga * __builtin_amdgcn_logf(ln)) : powf(ln, ga));
      }
    }
    if (!valid) scale = 0.f;
    c = scale * (1.0f / sqrtf((float)D));
    a = (g.alpha - 1.0f) * fabsf(c);
    w = 0.f;  // (see bias_w() in common.hip.h)
    if (g.slopes) {
      const float m = valid ? g.slopes[head] : 0.f;
      if (m != 0.f && a != 0.f) w = g.bias_mode == 0 ? (c < 0.f ? m : -m) * sqrtf((float)D) : -(g.alpha - 1.0f) * m / a;
    }
    if (a == 0.f) {
      a = 1.0f;
      c = 0.f;
    }
  }
  // d_ij from the dot product, without the bias
  __device__ __forceinline__ float signed_dot(float d) const { return c < 0.f ? -d : (c == 0.f ? 0.f : d); }
  __device__ __forceinline__ SeqRow of_lane(int l) const {
    SeqRow x;
    x.t = __shfl(t, l);
    x.head = __shfl(head, l);
    x.valid = __shfl(valid ? 1 : 0, l) != 0;
    x.lim = __shfl(lim, l);
    x.pos = __shfl(pos, l);
    x.a = __shfl(a, l);
    x.c = __shfl(c, l);
    x.w = __shfl(w, l);
    return x;
  }
};

// A wave's 32 rows, one to a lane pair, with the query fragments.
template <typename T, int D>
struct SeqRows : SeqRow {
  static constexpr int NC = D / 16;
  int lane, li, hh;
  int lim_min, lim_max; // over the wave's rows
  bool biased;          // some row of the wave has w != 0
  Frag<T> qf[NC];

  // rows r0 .. r0 + 31 of key/value head hk
  __device__ __forceinline__ void init(const SeqGeom& g, const SeqView& v, const void* Q, int hk, int r0) {
    lane = threadIdx.x & 63;
    li = lane & 31;
    hh = lane >> 5;
    SeqRow::init<sizeof(T) == 2>(g, v, hk, r0 + li, D);
    // (limits do not decrease from row to row)
    lim_min = __builtin_amdgcn_readfirstlane(lim);
    const int last = min(v.n * g.G - 1 - r0, 31);
    lim_max = last < 0 ? 0 : __builtin_amdgcn_readlane(lim, last);
    biased = __ballot(w != 0.f) != 0ull;
    const T* q = reinterpret_cast<const T*>(Q) + (long long)(v.row0 + t) * g.q_st + (long long)head * g.q_sh;
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) {
      Frag<T> f = c != 0.f ? Elem<T>::load(q + 16 * cc + 8 * hh) : Elem<T>::zero();  // (0 beyond the last row, too)
      qf[cc] = c < 0.f ? Elem<T>::negate(f) : f;
    }
  }
  __device__ __forceinline__ int key_of(int e) const { return 8 * (e >> 2) + 4 * hh + (e & 3); }
  // accumulator start of the 32 keys from j0 on
  __device__ __forceinline__ f32x16_t start(int j0) const {
    f32x16_t acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (biased) {
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = w * (float)max(pos - j0 - key_of(e), 0);
    }
    return acc;
  }
  // S^T of 32 keys whose fragments frag(cc) gives, on top of acc.  fp32: sums of eight features each, added up as a tree, because the rounding of these
  // sums is what the output's error comes from (one row against 1001 keys, D 64, four inputs: output off by 1.1e-7 to 8.3e-7, 3.7e-7 to 1.3e-6 with
  // plain matrix products; with four sums of sixteen features it was up to 1.1e-6).
  template <class F>
  __device__ __forceinline__ f32x16_t dots(f32x16_t acc, F frag) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) acc = Elem<T>::mma(frag(cc), qf[cc], acc);
      return acc;
    } else {
      return acc + tree<0, NC>(frag);
    }
  }
  template <int FROM, int N, class F>
  __device__ __forceinline__ f32x16_t tree(F frag) const {
    if constexpr (N > 1) {
      const f32x16_t left = tree<FROM, N / 2>(frag), right = tree<FROM + N / 2, N / 2>(frag);
      return left + right;
    } else {
      const Frag<T> f = frag(FROM);
      f32x16_t x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(f.lo[e], qf[FROM].lo[e], x, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_32x32x2f32(f.hi[e], qf[FROM].hi[e], y, 0, 0, 0);
      return x + y;
    }
  }
  // keys of the block at j0 that the row does not see; with holes, those on pages that are none as well
  __device__ __forceinline__ void mask(f32x16_t& acc, int j0, const SeqKeys& k, bool holes) const {
    const int rel = lim - j0;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = key_of(e) < rel ? acc[e] : -kInf;
    if (holes) {
#pragma unroll 1
      for (int e = 0; e < 16; ++e) {
        const bool out = key_of(e) < rel && k.is_hole(k.page(j0 + key_of(e)));
#pragma unroll
        for (int u = 0; u < 16; ++u)
          if (u == e && out) acc[u] = -kInf;
      }
    }
  }
};

}  // namespace entmax
