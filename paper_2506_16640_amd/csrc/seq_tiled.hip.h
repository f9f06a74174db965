// Entmax attention of packed sequences over packed or paged keys, any density: one workgroup per 128 folded rows of a
// key/value head (SeqRows), key tiles through LDS, scores recomputed by every sweep (S^T = K Q^T, a lane owns a row):
//   1. bounds and a starting point for the threshold tau of
//        f(tau) = sum_j [y_j - tau]_+^r - 1 = 0,   y = (alpha-1) s,  r = 1 / (alpha-1)
//      from the list kernels, or from a sample of the key tiles
//   2. sweeps over K that evaluate f and step (SeqSearch); the first one notes which 32-key blocks can hold a positive term at all
//   3. a sweep over K and V: O^T = V^T P^T on the matrix cores.  The accumulators of S^T are the second operand as they are; V^T comes out
//      of row-major tiles through transposing LDS reads (ds_read_b64_tr_b16: sixteen lanes give four rows of sixteen
//      elements, each lane gets a column), so that no transposed copy of V exists anywhere.
// A block's sweeps follow one another, and few blocks may be left to this kernel: so a block has 8 or 16 waves, and KS of them share the
// keys of each tile for the same 32 rows (their sums are added in their order).
// Measured: 6 prompts of 300 to 2000 tokens, 4 x 4 heads of 128, logits without a scale: 189 us, of it starts and ends 18, the first evaluation 35, later
// ones 61, P V 74 (all sweeps bound by the vector work on the scores: the products are 10 us at the rate of a large one).
#pragma once
#include "fwd.hip.h"
#include "seq.hip.h"
#include "seq_layout.h"
#include "seq_search.h"

namespace entmax {

// What the sweep of the list kernels leaves of a group of 128 rows, so that nobody has to look for its sequence again
struct SeqBlock {
  int s, row0, n, L, r0;  // the sequence (see SeqView; s = -1: nothing to do) and the group's first folded row
};

struct SeqArgs {
  SeqGeom g;
  const void* Q;
  const void* K;
  const void* V;
  void* O;
  int nblk;        // 128-row groups per key/value head (seq_blocks())
  int mark_shift, mark_words;  // seq_tiled_kernel: a word of marks for every 1 << mark_shift key tiles
  const int* dense;  // NULL, or [Hkv * nblk]: only the groups that are marked, kFlagDense or kFlagWithBounds
  const SeqBlock* blocks;  // with dense: [Hkv * nblk]
  const float2* bounds;  // with dense: [Hkv * nblk][128] of groups with bounds: (lower bound of the threshold relative to the largest y, largest raw score)
  int split;       // sequences with few rows are left to the kernels that split the keys
};

// Whether the kernels that split the keys take a sequence (else those for 128 rows at a time do)
__device__ __forceinline__ bool split_seq(const SeqGeom& g, const SeqView& v) { return (long long)v.n * g.G <= kSplitRows; }


// Group blk of 128 rows: its sequence and its first folded row; false: nothing to do.
__device__ __forceinline__ bool seq_block(const SeqGeom& g, int blk, bool split, SeqView& v, int& r0) {
  // sequence s has the groups from cu[s] G / 128 + s on
  const int G = g.G;
  auto first = [G](int c, int s) { return (long long)c * G / kBlockRows + s; };
  const int s = find_seq(g.cu, g.nseq, blk, first);
  r0 = 0;
  if (s >= g.nseq || !load_seq(g, s, v) || (split && split_seq(g, v))) return false;
  const long long local = blk - first(v.row0, s);
  if (local < 0 || local * kBlockRows >= (long long)v.n * G) return false;
  r0 = (int)local * kBlockRows;
  return true;
}

// WIDE: KS waves share the keys of 32 rows, one workgroup fills a compute unit; else a workgroup of four waves, two or more to a unit.
template <typename T, int D, bool WIDE>
struct SeqTiledCfg {
  static constexpr int KS = !WIDE || (sizeof(T) == 4 && D == 128) ? 1 : (sizeof(T) == 2 && D == 64 ? 4 : 2);
  static constexpr int NT = KS * kThreads;
  static constexpr int kWavesPerSimd = sizeof(T) == 2 && D == 64 ? (WIDE ? 4 : 3) : (sizeof(T) == 4 && D == 128 ? 1 : 2);
  static constexpr int BW = sizeof(T) == 4 && D == 128 ? 1 : 2;      // 32-key blocks of a wave per tile
  static constexpr int KT = KS * BW * 32;
  static constexpr int kTileBytes = KT * D * (int)sizeof(T);
  static_assert(kTileBytes <= 32768, "four tiles and the marks fit a compute unit");
  static size_t lds_bytes(int mark_words) { return 4 * (size_t)kTileBytes + (size_t)mark_words * 4; }
};

// Adds a block of a lane's scores to the sums at tau (relative to the row's largest score, a ref), x = [y - tau]_+ at most 1, for tau is never below the
// largest y by more: the clamp of the multiply-add is the lower and the upper limit in one.  CURV: k too (alpha 1.5: the count; alpha 2 and
// general alpha: not formed).  The difference of the scores is exact where it counts: scores of a few thousand lose no bits of the probabilities.
template <int AM, bool CURV>
__device__ __forceinline__ void accumulate_keys(SeqSums& s, const f32x16_t& acc, float ref, float a, float tau, float r) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float x = __builtin_amdgcn_fmed3f(fmaf(acc[e] - ref, a, -tau), 0.f, 1.f);
    if (AM == 1) {
      s.g += x;
      s.h = fmaf(x, x, s.h);
      if (CURV) s.k += x > 0.f ? 1.f : 0.f;
    } else if (AM == 2) {
      s.h += x;
      s.g += x > 0.f ? 1.f : 0.f;
    } else if (AM == 3) {
      const float x2 = x * x;
      s.g = fmaf(x2, x, s.g);
      s.h = fmaf(x2, x2, s.h);
      if (CURV) s.k += x2;
    } else if (x > 0.f) {
      const float l = __builtin_amdgcn_logf(x);
      s.h += __builtin_amdgcn_exp2f(r * l);
      s.g += __builtin_amdgcn_exp2f((r - 1.f) * l);
    }
  }
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 read_transposed(const char* lds) {
  const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)lds);
  return __builtin_bit_cast(uint2, v);
}

// Fragments of V^T for the product that contracts over the 16 keys 16 c .. 16 c + 15 of a 32-key block, in the order of the accumulators:
// element e of half hh is key 16 c + 8 (e / 4) + 4 hh + e % 4.
template <typename T, int D, int KT, int NT = kThreads>
struct SeqValues {
  static constexpr int NM = D / 32;
  using VT = SeqTile<T, D, KT, sizeof(T) == 2, NT>;
  int voff[NM];
  int li, hh;
  __device__ __forceinline__ void init(int lane) {
    li = lane & 31;
    hh = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int p = lane & 15, row = 4 * hh + (p >> 2);
#pragma unroll
      for (int mm = 0; mm < NM; ++mm)
        voff[mm] = VT::off(row, 4 * mm + 2 * ((lane >> 4) & 1) + ((p & 3) >> 1)) + (p & 1) * 8;
    }
  }
  __device__ __forceinline__ Frag<T> frag(const char* vt, int sb, int c, int mm) const {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      const char* at = vt + voff[mm] + (sb * 32 + 16 * c) * VT::kRowBytes;
      const uint2 x = read_transposed(at), y = read_transposed(at + 8 * VT::kRowBytes);
      f.v = u32x4_t{x.x, x.y, y.x, y.y};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = value(vt, sb * 32 + 16 * c + 8 * (e >> 2) + 4 * hh + (e & 3), 32 * mm + li);
        if (e < 4) f.lo[e] = x; else f.hi[e - 4] = x;
      }
    }
    return f;
  }
  static __device__ __forceinline__ float value(const char* vt, int row, int feature) {
    constexpr int E = 16 / (int)sizeof(T);
    const char* at = vt + VT::off(row, feature / E) + (feature % E) * (int)sizeof(T);
    if constexpr (sizeof(T) == 2)
      return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16);
    else
      return *reinterpret_cast<const float*>(at);
  }
  static __device__ __forceinline__ bool not_finite(const Frag<T>& f) {
    bool bad = false;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) bad = bad || (f.v[k] & 0x7f80u) == 0x7f80u || (f.v[k] & 0x7f800000u) == 0x7f800000u;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        bad = bad || (__float_as_uint(f.lo[k]) & 0x7f800000u) == 0x7f800000u || (__float_as_uint(f.hi[k]) & 0x7f800000u) == 0x7f800000u;
    }
    return bad;
  }
  // oacc += V^T P^T of block sb.  special: some row does not see some key of the block (then 0 x infinity must not come in: where a value is not finite,
  // the products with non-zero probabilities are formed one by one).
  __device__ __forceinline__ void accumulate(const char* vt, int sb, const float (&p)[16], bool special, f32x16_t (&oacc)[NM]) const {
    if (special) {
      bool bad = false;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int mm = 0; mm < NM; ++mm) bad = not_finite(frag(vt, sb, c, mm)) || bad;
      if (__ballot(bad) != 0ull) {
        one_by_one(vt, sb, p, oacc);
        return;
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      // the probabilities as the sum of two bf16 numbers: rounded to one, they would cost up to 2^-9 |v| of the output
      Frag<T> ph, pl;
      Elem<T>::pack_split(p + 8 * c, ph, pl);
#pragma unroll
      for (int mm = 0; mm < NM; ++mm) {
        const Frag<T> v = frag(vt, sb, c, mm);
        oacc[mm] = Elem<T>::mma(v, ph, oacc[mm]);
        if constexpr (Elem<T>::kSplit) oacc[mm] = Elem<T>::mma(v, pl, oacc[mm]);
      }
    }
  }
  __device__ __forceinline__ void one_by_one(const char* vt, int sb, const float (&p)[16], f32x16_t (&oacc)[NM]) const {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float other = __shfl_xor(p[e], 32);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float pk = half == hh ? p[e] : other;
        if (pk > 0.f) {
          const int row = sb * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
#pragma unroll
          for (int mm = 0; mm < NM; ++mm)
#pragma unroll
            for (int x = 0; x < 16; ++x)
              oacc[mm][x] = fmaf(pk, value(vt, row, 32 * mm + 8 * (x >> 2) + 4 * hh + (x & 3)), oacc[mm][x]);
        }
      }
    }
  }
};

// Four consecutive features of a lane's row, in the type of O
template <typename T>
__device__ __forceinline__ void store4(T* dst, float x0, float x1, float x2, float x3) {
  if constexpr (sizeof(T) == 2) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    const bf16x4_t b = {(__bf16)x0, (__bf16)x1, (__bf16)x2, (__bf16)x3};
    *reinterpret_cast<uint2*>(dst) = __builtin_bit_cast(uint2, b);
  } else {
    *reinterpret_cast<f32x4_t*>(dst) = f32x4_t{x0, x1, x2, x3};
  }
}

template <typename T, int D, int AM, bool WIDE>
__global__ __launch_bounds__((SeqTiledCfg<T, D, WIDE>::NT), (SeqTiledCfg<T, D, WIDE>::kWavesPerSimd)) void seq_tiled_kernel(SeqArgs A) {
  using Cfg = SeqTiledCfg<T, D, WIDE>;
  constexpr int NT = Cfg::NT, KS = Cfg::KS, BW = Cfg::BW, KT = Cfg::KT, NSB = KT / 32, NC = D / 16, NM = D / 32, TB = Cfg::kTileBytes;
  using KTile = SeqTile<T, D, KT, false, NT>;
  using Vals = SeqValues<T, D, KT, NT>;
  using VTile = typename Vals::VT;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const SeqGeom& g = A.g;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rg = wave & 3, ks = wave >> 2;
  // The head runs fastest, so that a head's groups meet on one XCD where the heads divide among the eight of them; the groups run from the
  // last to the first, a sequence's long rows first.
  const int hk = blockIdx.x % g.Hkv, blk = A.nblk - 1 - (int)blockIdx.x / g.Hkv;
  const int flag = A.dense ? A.dense[hk * A.nblk + blk] : kFlagDense;
  if (flag == 0) return;
  SeqView v;
  int blk0;
  if (A.dense) {
    const SeqBlock b = A.blocks[hk * A.nblk + blk];
    v = SeqView{b.s, b.row0, b.n, b.L};
    blk0 = b.r0;
  } else if (!seq_block(g, blk, A.split != 0, v, blk0)) {  // (the same for the whole workgroup)
    return;
  }
  SeqKeys keys, vals;
  keys.init(g, v, A.K, hk, false, sizeof(T));
  vals.init(g, v, A.V, hk, true, sizeof(T));
  SeqRows<T, D> q;
  q.init(g, v, A.Q, hk, blk0 + rg * 32);
  const int last_row = min(v.n * g.G, blk0 + kBlockRows) - 1;
  const int block_lim = g.causal ? max(0, min(v.L - v.n + last_row / g.G + 1, v.L)) : v.L;
  const int ntiles = __builtin_amdgcn_readfirstlane((block_lim + KT - 1) / KT);
  const bool holes = seq_has_holes(keys, block_lim);
  const float r = 1.0f / (g.alpha - 1.0f);
  const int lane = q.lane;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  // which blocks can hold a positive term for some row of a row group, noted in the first sweep over all keys: bit
  // 8 (row group) + (block of the tile) of the tile's word
  static_assert(NSB <= 8, "eight bits a row group");
  uint32_t* marks = reinterpret_cast<uint32_t*>(smem + 4 * TB);
  for (int w = threadIdx.x; w < A.mark_words; w += NT) marks[w] = 0u;
  auto marks_of = [&](int kt) { return (uint32_t)__builtin_amdgcn_readfirstlane(marks[kt >> A.mark_shift]); };
  auto tile_marked = [&](int kt) { return marks_of(kt) != 0u; };

  FragOff<T> koff[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc) koff[cc] = FragOff<T>::template make<typename KTile::Tile>(q.li, 2 * cc + q.hh);
  auto next = [&](int kt, auto needed) {
    while (kt < ntiles && !needed(kt)) ++kt;
    return kt;
  };
  // K tiles kt with needed(kt) (uniform), three of them under way while one is worked on: body(kt, tile)
  auto sweep_k = [&](auto needed, auto body) {
    typename KTile::Pages pg;
    auto issue = [&](int t, int buf) { KTile::load(keys, pg, t * KT, v.L, lds0 + (uint32_t)buf * TB, wave, lane); };
    int t0 = next(0, needed), t1 = ntiles, t2 = ntiles, t3 = ntiles;
    __syncthreads();  // (the tile buffers are free)
    if (t0 < ntiles) {
      pg.ask(keys, t0 * KT, v.L, wave);
      issue(t0, 0);
      t1 = next(t0 + 1, needed);
    }
    if (t1 < ntiles) {
      pg.ask(keys, t1 * KT, v.L, wave);
      issue(t1, 1);
      t2 = next(t1 + 1, needed);
    }
    if (t2 < ntiles) {
      pg.ask(keys, t2 * KT, v.L, wave);
      issue(t2, 2);
      t3 = next(t2 + 1, needed);
      if (t3 < ntiles) pg.ask(keys, t3 * KT, v.L, wave);
      lds_loads_wait<2 * KTile::L>();
    } else if (t1 < ntiles) {
      lds_loads_wait<KTile::L>();
    } else {
      lds_loads_wait<0>();
    }
    __syncthreads();
    int cur = 0;
    while (t0 < ntiles) {
      int t4 = ntiles;
      if (t3 < ntiles) {
        issue(t3, (cur + 3) & 3);  // that of the tile before, which every wave has left
        t4 = next(t3 + 1, needed);
        if (t4 < ntiles) pg.ask(keys, t4 * KT, v.L, wave);
      }
      body(t0, smem + cur * TB);
      if (t3 < ntiles)
        lds_loads_wait<2 * KTile::L>();
      else if (t2 < ntiles)
        lds_loads_wait<KTile::L>();
      else
        lds_loads_wait<0>();
      __syncthreads();
      cur = (cur + 1) & 3;
      t0 = t1;
      t1 = t2;
      t2 = t3;
      t3 = t4;
    }
  };
  // fn(acc, block of the tile, masked) on the scores of this wave's blocks of the tile that some row of it sees; with `only_marked` of those
  // that are marked
  auto each_block = [&](int kt, const char* tl, bool only_marked, auto fn) {
    const uint32_t bits = only_marked ? marks_of(kt) >> (8 * rg) : ~0u;
#pragma unroll 1
    for (int b = 0; b < BW; ++b) {
      const int sb = ks * BW + b, j0 = kt * KT + sb * 32;
      if (j0 >= q.lim_max || ((bits >> sb) & 1u) == 0u) continue;
      const char* at = tl + sb * 32 * KTile::kRowBytes;
      f32x16_t acc = q.dots(q.start(j0), [&](int cc) { return koff[cc].load(at, 0); });
      const bool masked = holes || j0 + 32 > q.lim_min;
      if (masked) q.mask(acc, j0, keys, holes);
      fn(acc, sb, masked);
    }
  };
  // Exchange between the waves that share the row group's keys (in the tile buffers, which are free between sweeps).
  f32x4_t* xch = reinterpret_cast<f32x4_t*>(smem);
  auto post = [&](const f32x4_t& x) {
    xch[wave * 64 + lane] = x;
    __syncthreads();
  };

  // ------------------------------------------------------------ 1. where to start
  // (y, tau and the bracket are relative to a ref, the largest score known; the whole search is)
  const bool given = flag == kFlagWithBounds;
  float m = -kInf, ref = 0.f, lo = -1.f, hi = kInf, tau = -1.f;
  const float below = q.lim > 0 ? __builtin_amdgcn_exp2f(-(g.alpha - 1.0f) * __builtin_amdgcn_logf((float)q.lim)) : 1.f;
  bool live, know_max = true;
  if (given) {
    const float2 bd = A.bounds[((long long)hk * A.nblk + blk) * kBlockRows + rg * 32 + q.li];
    live = q.lim > 0 && bd.y > -3.0e38f;  // (-3e38: the list kernels' score of masked keys)
    ref = live ? bd.y : 0.f;
    hi = -below;
    lo = live ? fminf(fmaxf(-1.0f, bd.x), hi) : -1.0f;
    tau = lo;
  } else {
    // a sample of about four tiles (all of them where there are no more, and where a tile may show a row no key at all)
    const int every = holes ? 1 : max(1, ntiles >> 2);
    float ms1 = 0.f, ms2 = 0.f, msn = 0.f;
    sweep_k([&](int kt) { return kt % every == 0; },
            [&](int kt, const char* tl) {
              each_block(kt, tl, false, [&](f32x16_t& acc, int, bool masked) {
                if (!masked && AM != 0) {
#pragma unroll
                  for (int e = 0; e < 16; ++e) {
                    ms1 += acc[e];
                    ms2 = fmaf(acc[e], acc[e], ms2);
                  }
                  msn += 32.f;
                }
                m = fmaxf(m, max16(acc));
              });
            });
    m = fmaxf(m, __shfl_xor(m, 32));
    ms1 += __shfl_xor(ms1, 32);
    ms2 += __shfl_xor(ms2, 32);
    post(f32x4_t{m, ms1, ms2, msn});
    ms1 = ms2 = msn = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const f32x4_t x = xch[(4 * k + rg) * 64 + lane];
      m = fmaxf(m, x[0]);
      ms1 += x[1];
      ms2 += x[2];
      msn += x[3];
    }
    live = q.lim > 0 && m > -kInf;
    know_max = every == 1;
    ref = live ? m : 0.f;  // (the largest score is at least the sample's)
    if (know_max) hi = -below;
    if (live && msn >= 64.f) {
      const float mean = ms1 / msn, var = ms2 / msn - mean * mean;
      float t0;
      if (var > 0.f && gauss_start<AM>(q.a * (mean - ref), q.a * sqrtf(var), (float)q.lim, t0)) tau = fminf(fmaxf(t0, lo), hi);
    }
  }
  const float lo0 = lo, ref0 = ref;  // blocks without a term above lo0 are zero for good

  // ------------------------------------------------------------ 2. threshold
  SeqSearch<AM> search{tau, lo, hi, (float)q.lim, 0.f, 0.f, 0.f, false, false};
  bool done = !live;
  int iter = 0, more;
  auto sweep = [&](auto first_) {
    constexpr bool FIRST = decltype(first_)::value;
    const bool wave_on = __ballot(!done) != 0ull;
    SeqSums sums{0.f, 0.f, 0.f};
    const float t_now = done ? kInf : search.tau;
    sweep_k([&](int kt) { return FIRST || tile_marked(kt); },
            [&](int kt, const char* tl) {
              if (!wave_on) return;
              each_block(kt, tl, !FIRST, [&](f32x16_t& acc, int sb, bool masked) {
                if (FIRST) {
                  const float lm = max16(acc);
                  m = fmaxf(m, lm);
                  const bool any = live && lm > -kInf && fmaf(lm - ref0, q.a, -lo0) > 0.f;
                  if (__ballot(any) == 0ull) return;
                  if (lane == 0) atomicOr(&marks[kt >> A.mark_shift], 1u << (8 * rg + sb));
                }
                accumulate_keys<AM, FIRST>(sums, acc, ref, q.a, t_now, r);
              });
            });
    sums.g += __shfl_xor(sums.g, 32);
    sums.h += __shfl_xor(sums.h, 32);
    sums.k += __shfl_xor(sums.k, 32);
    if (FIRST) m = fmaxf(m, __shfl_xor(m, 32));
    post(f32x4_t{sums.g, sums.h, sums.k, m});
    sums = SeqSums{0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const f32x4_t x = xch[(4 * k + rg) * 64 + lane];
      sums.g += x[0];
      sums.h += x[1];
      sums.k += x[2];
      if (FIRST) m = fmaxf(m, x[3]);
    }
    if (FIRST && !know_max) {
      // from the sample's largest score to the row's
      const float up = live ? q.a * (m - ref) : 0.f;
      ref = live ? m : 0.f;
      search.tau -= up;
      search.lo = fmaxf(search.lo - up, -1.0f);
      search.hi = -below;
    }
    if (!done) done = search.step(sums, r, FIRST && (AM == 1 || AM == 3));
    ++iter;
    more = __syncthreads_or(done ? 0 : 1);
  };
  sweep(std::true_type());
  while (more && iter < kMaxSolveIters) sweep(std::false_type());
  tau = search.tau;

  // ------------------------------------------------------------ 3. O^T = V^T P^T
  f32x16_t oacc[NM];
#pragma unroll
  for (int mm = 0; mm < NM; ++mm)
    oacc[mm] = f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  Vals vv;
  vv.init(lane);
  const float t_out = live ? tau : kInf;
  {
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
    int t0 = next(0, tile_marked), t1 = ntiles;
    if (t0 < ntiles) {
      ask(t0);
      issue(t0, 0);
      t1 = next(t0 + 1, tile_marked);
      if (t1 < ntiles) ask(t1);
    }
    lds_loads_wait<0>();
    __syncthreads();
    int cur = 0;
    while (t0 < ntiles) {
      int t2 = ntiles;
      if (t1 < ntiles) {
        issue(t1, cur ^ 1);
        t2 = next(t1 + 1, tile_marked);
        if (t2 < ntiles) ask(t2);
      }
      const char* tl = smem + cur * 2 * TB;
      each_block(t0, tl, true, [&](f32x16_t& acc, int sb, bool masked) {
        float p[16], any = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          p[e] = pow_r<AM>(__builtin_amdgcn_fmed3f(fmaf(acc[e] - ref, q.a, -t_out), 0.f, 1.f), r);
          any = fmaxf(any, p[e]);
        }
        if (__ballot(any > 0.f) == 0ull) return;  // every probability of the block is zero
        vv.accumulate(tl + TB, sb, p, masked, oacc);
      });
      lds_loads_wait<0>();
      __syncthreads();
      cur ^= 1;
      t0 = t1;
      t1 = t2;
    }
  }
  // the sums of the waves that shared the keys, each of them adding up its part of the features
  f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);  // [waves][NM * 4][64]
#pragma unroll
  for (int mm = 0; mm < NM; ++mm)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      red[(wave * NM * 4 + mm * 4 + x) * 64 + lane] = f32x4_t{oacc[mm][4 * x], oacc[mm][4 * x + 1], oacc[mm][4 * x + 2], oacc[mm][4 * x + 3]};
  __syncthreads();
  if (!q.valid) return;
  T* o = reinterpret_cast<T*>(A.O) + (long long)(v.row0 + q.t) * g.o_st + (long long)q.head * g.o_sh;
  constexpr int PER = NM * 4 / KS;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int f = ks * PER + u;  // features 32 (f / 4) + 8 (f % 4) + 4 hh on
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const f32x4_t x = red[((4 * k + rg) * NM * 4 + f) * 64 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    store4<T>(o + 8 * f + 4 * q.hh, sum[0], sum[1], sum[2], sum[3]);
  }
}

}  // namespace entmax
