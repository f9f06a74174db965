// Serving attention for 128 folded rows at a time where supports are short: one sweep over the keys, then only the keys that can matter.
//   seq_sweep_kernel   S^T = K Q^T with K tiles straight to LDS; every lane (half a row) keeps its largest groups of eight keys
//                      (TopGroups, fwd_sparse.hip.h) and its largest score, and leaves them in the workspace.  A group of rows may be
//                      shared out to several workgroups by keys where there are few of them.
//   seq_finish_kernel  eight lanes (an octet) per row: a lower bound of the threshold from the groups' largest scores, the scores of the groups
//                      above it once more from memory (each lane then holds one key of every group), threshold, and the output from the
//                      values of the support.  Rows that remember too few groups are looked through key by key; where a block has many of
//                      those, or its rows are dense, it is left to seq_tiled_kernel.
// Measured: 4 x 512 tokens, 4 x 4 heads of 128, against 2000 to 16384 keys: sweep 96 us (650 TFLOP/s: the vector work on the scores beside the matrix
// work; 186 us without sharing out the keys), finish 49 to 54 us (dependent gathers: groups, keys, values).
#pragma once
#include "decode.hip.h"
#include "fwd_sparse.hip.h"
#include "seq.hip.h"
#include "seq_tiled.hip.h"

namespace entmax {

constexpr int kTopWords = kTopGroups + 2;  // of a lane: its groups, its largest score, how many of the groups were kept throughout
static_assert(kTopWords == kSeqTopWords, "the workspace holds them");

struct SeqListArgs {
  SeqArgs a;
  SeqBlock* blocks;  // [Hkv * nblk]
  float* tops;       // [Hkv * nblk][ksplit][4 waves][kTopWords][64]
  int* votes;        // [Hkv * nblk][ksplit] 1: the rows are dense
  int* dense;        // [Hkv * nblk] kFlagDense, kFlagWithBounds: left to seq_tiled_kernel (with the rows' bounds)
  float2* bounds;    // [Hkv * nblk][128]
  int ksplit;        // workgroups that share the keys of a block
};

template <int D>
struct SeqSweepCfg {
  static constexpr int KT = D == 64 ? 128 : 64;
  static constexpr int kTileBytes = KT * D * 2;
  static constexpr size_t kLdsBytes = 3 * (size_t)kTileBytes + 16;
};

template <int D>
__global__ __launch_bounds__(kThreads, 3) void seq_sweep_kernel(SeqListArgs A) {
  using T = bf16_t;
  using Cfg = SeqSweepCfg<D>;
  constexpr int KT = Cfg::KT, NSB = KT / 32, NC = D / 16, TB = Cfg::kTileBytes, G8 = 8;
  using KTile = SeqTile<T, D, KT, false>;
  using Top = TopGroups<G8>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  int* votes = reinterpret_cast<int*>(smem + 3 * TB);
  const SeqGeom& g = A.a.g;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int item = blockIdx.x / A.ksplit, part = blockIdx.x % A.ksplit;
  const int hk = item % g.Hkv, blk = A.a.nblk - 1 - item / g.Hkv;
  const int id = hk * A.a.nblk + blk;
  SeqView v;
  int r0;
  const bool mine = seq_block(g, blk, A.a.split != 0, v, r0);
  if (part == 0 && threadIdx.x == 0) {
    A.blocks[id] = SeqBlock{mine ? v.s : -1, v.row0, v.n, v.L, r0};
    A.dense[id] = 0;
  }
  if (!mine) return;
  if (threadIdx.x < 4) votes[threadIdx.x] = 0;  // (before the first barrier)
  SeqKeys keys;
  keys.init(g, v, A.a.K, hk, false, sizeof(T));
  SeqRows<T, D> q;
  q.init(g, v, A.a.Q, hk, r0 + wave * 32);
  const int lane = q.lane;
  const int last_row = min(v.n * g.G, r0 + kBlockRows) - 1;
  const int first_lim = g.causal ? max(0, min(v.L - v.n + r0 / g.G + 1, v.L)) : v.L;  // (limits do not decrease)
  const int block_lim = g.causal ? max(0, min(v.L - v.n + last_row / g.G + 1, v.L)) : v.L;
  const int all_tiles = (block_lim + KT - 1) / KT, share = (all_tiles + A.ksplit - 1) / A.ksplit;
  const int first = __builtin_amdgcn_readfirstlane(min(part * share, all_tiles));
  const int ntiles = __builtin_amdgcn_readfirstlane(min(first + share, all_tiles));
  const bool holes = seq_has_holes(keys, block_lim);
  // tiles before this one are seen whole by every row, and with a distance bias lie before every row's position
  const bool biased = g.slopes != nullptr;
  const int whole_end = holes || (biased && !g.causal) ? first : __builtin_amdgcn_readfirstlane(min(first_lim / KT, ntiles));
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  FragOff<T> koff[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc) koff[cc] = FragOff<T>::template make<typename KTile::Tile>(q.li, 2 * cc + q.hh);
  auto scores = [&](const char* tl, int sb, int kt) {
    f32x16_t acc = q.start(kt * KT + sb * 32);
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) acc = Elem<T>::mma(koff[cc].load(tl, sb * 32 * KTile::kRowBytes), q.qf[cc], acc);
    return acc;
  };

  const GroupNumbers<G8> gn(max(v.L, 1));
  Top top;
  top.init();
  float m1 = -kInf;
  int kt = first, cur = 0;
  typename KTile::Pages pg;
  auto issue = [&](int t, int buf) { KTile::load(keys, pg, t * KT, v.L, lds0 + (uint32_t)buf * TB, wave, lane); };
  if (kt < ntiles) {
    pg.ask(keys, kt * KT, v.L, wave);
    issue(kt, 0);
  }
  if (kt + 1 < ntiles) {
    pg.ask(keys, (kt + 1) * KT, v.L, wave);
    issue(kt + 1, 1);
    pg.ask(keys, (kt + 2) * KT, v.L, wave);  // (a place behind the last tile is asked for at the last key)
    lds_loads_wait<KTile::L>();
  } else {
    lds_loads_wait<0>();
  }
  __syncthreads();
  // body(tile) on tile kt; two more are under way
  auto step = [&](auto body) {
    const bool more = kt + 2 < ntiles;
    if (more) {
      issue(kt + 2, cur == 0 ? 2 : cur - 1);  // that of the tile before, which every wave has left
      pg.ask(keys, (kt + 3) * KT, v.L, wave);
    }
    body(smem + cur * TB);
    if (more)
      lds_loads_wait<KTile::L>();
    else
      lds_loads_wait<0>();
    __syncthreads();
    cur = cur == 2 ? 0 : cur + 1;
    ++kt;
  };
  auto general = [&](const char* tl) {
#pragma unroll 1
    for (int sb = 0; sb < NSB; ++sb) {
      const int j0 = kt * KT + sb * 32;
      if (j0 >= q.lim_max) break;
      f32x16_t acc = scores(tl, sb, kt);
      if (holes || j0 + 32 > q.lim_min) q.mask(acc, j0, keys, holes);
      m1 = fmaxf(m1, top.take(acc, gn, j0 >> 5));
    }
  };
  // Dense rows show on the first tile: for three quarters of a wave's rows nearly all keys of the first block come within the
  // threshold's reach of the block's largest score.  If all waves find so the block is seq_tiled_kernel's, which then starts from a sample.  (Rows of
  // fewer candidates get better bounds from this sweep than the sample gives, and save it more than the sweep takes.)
  if (first < whole_end) {
    const f32x16_t acc = scores(smem, 0, first);
    const float lm = max16(acc);
    const float reach = q.lim > 0 ? (q.a > 0.f ? 1.0001f / q.a : 3.0e38f) : -kInf;
    int near = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) near += (acc[e] + reach > lm) ? 1 : 0;
    const bool dense = 4 * (int)__popcll(__ballot(near >= 15)) >= 3 * (int)__popcll(__ballot(q.lim > 0));
    if (dense && lane == 0) votes[wave] = 1;
    __syncthreads();
  }
  const bool all_dense = (votes[0] & votes[1] & votes[2] & votes[3]) != 0;
  if (threadIdx.x == 0) A.votes[(long long)id * A.ksplit + part] = all_dense ? 1 : 0;
  if (all_dense) {
    lds_loads_wait<0>();
    return;
  }
  // Tiles all of whose keys every row sees: the matrix instructions of a block run beside the vector work on the scores of the one before it
  // (the same interleaving as in fwd_lists_blocks(), fwd_sparse.hip.h)
  auto whole_tiles = [&](auto biased_, auto places_) {
    constexpr int K = decltype(places_)::value;
    f32x16_t late;
#pragma unroll
    for (int e = 0; e < 16; ++e) late[e] = -kInf;
    int late_jb = 0;
    float late_floor = Top::kNothing;  // (nothing waits)
    auto pipelined = [&](const char* tl) {
      constexpr int F = 4;  // fragments in registers
      Frag<T> kf[F];
#pragma unroll
      for (int cc = 0; cc < F; ++cc) kf[cc] = koff[cc].load(tl, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb) {
        const int j0 = kt * KT + sb * 32;
        float m[Top::Numbers::kPerBlock], x[Top::Numbers::kPerBlock];
        f32x16_t acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if constexpr (decltype(biased_)::value) {
          const float base = q.w * (float)(q.pos - j0 - 4 * q.hh);
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[e] = fmaf(-q.w, (float)(8 * (e >> 2) + (e & 3)), base);
        }
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) {
          acc = Elem<T>::mma(kf[cc % F], q.qf[cc], acc);
          const int nx = cc + F;  // what this place holds next: a later fragment of the block, or one of the next block's
          if (nx < NC)
            kf[cc % F] = koff[nx].load(tl, sb * 32 * KTile::kRowBytes);
          else if (sb + 1 < NSB)
            kf[cc % F] = koff[nx - NC].load(tl, (sb + 1) * 32 * KTile::kRowBytes);
          __builtin_amdgcn_sched_barrier(0);
          if (cc == 0) top.template take_part<0, K>(late, gn, late_jb, late_floor, m, x, m1);
          if (cc == NC / 4) top.template take_part<1, K>(late, gn, late_jb, late_floor, m, x, m1);
          if (cc == 2 * NC / 4) top.template take_part<2, K>(late, gn, late_jb, late_floor, m, x, m1);
          if (cc == 3 * NC / 4) top.template take_part<3, K>(late, gn, late_jb, late_floor, m, x, m1);
          __builtin_amdgcn_sched_barrier(0);
        }
        late = acc;
        late_jb = j0 >> 5;
        late_floor = Top::kFloor;
      }
#pragma unroll
      for (int e = 0; e < K; ++e) asm volatile("" : "+v"(top.t[e]));
      asm volatile("" : "+v"(m1));
    };
#pragma unroll 1
    while (kt < whole_end) step(pipelined);
    m1 = fmaxf(m1, top.take(late, gn, late_jb, late_floor));
  };
  const bool weak = q.lim > 0 && !(q.a * sqrtf((float)D) >= kFewPlacesScale);
  const bool few = __ballot(weak) == 0ull;
  auto both = [&](auto biased_) {
    if (few)
      whole_tiles(biased_, std::integral_constant<int, kFewPlaces>());
    else
      whole_tiles(biased_, std::integral_constant<int, kTopGroups>());
  };
  if (kt < whole_end) {
    if (q.biased)
      both(std::true_type());
    else
      both(std::false_type());
  }
  while (kt < ntiles) step(general);
  float* dst = A.tops + (((long long)id * A.ksplit + part) * kWaves + wave) * (kTopWords * 64) + lane;
#pragma unroll
  for (int e = 0; e < kTopGroups; ++e) dst[e * 64] = top.t[e];
  dst[kTopGroups * 64] = m1;
  dst[(kTopGroups + 1) * 64] = few && first < whole_end ? (float)kFewPlaces : (float)kTopGroups;
}

// Octets: eight lanes work on a row, lane c with 16-byte word c of every 128 bytes of a key, value or query row.
template <int CTRL>
__device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false)));
}
template <int CTRL>
__device__ __forceinline__ float dpp_min(float x) {
  return fminf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float max8(float x) { return dpp_max<0x4E>(dpp_max<0xB1>(dpp_max<0x141>(x))); }
__device__ __forceinline__ float min8(float x) { return dpp_min<0x4E>(dpp_min<0xB1>(dpp_min<0x141>(x))); }

constexpr int kFinishSlots = 24;    // groups of a row that an octet can hold (eight keys each)
constexpr int kFinishSupport = 32;  // support entries of a row noted before their values are gathered
constexpr int kScanList = 256;      // candidates of a row that all octets look through together
// The rows that the finish kernel takes the long way instead of giving their whole block to the tiled kernel.  Blocks of 128 rows against 32000 keys,
// alpha 1.7, no scale: 59 us here and nothing left for the tiled kernel; with none taken 51 us here and 1720 us there.  Where blocks are dense
// anyway it costs time here (prompts of 300 to 2000 tokens without a scale: 46 us for 36; prompts with scales: 66 us for 62).  Rows looked through key by
// key are rarer: with none of them the first case leaves 4 us more to the tiled kernel, and with groups up to 200 instead of 40 the prompts without a
// scale cost 53 us here.
constexpr int kHardRows = 3;        // such rows of a wave (eight rows): with more groups than an octet holds, or (one of them) looked through key by key
constexpr int kScanGroups = 40;     // ... where the wave's other rows have at most so many groups together
constexpr int kScanKeys = 8192;     // ... and at most so many keys

template <int D>
struct OctetRow {  // of a key/value row or query: the lane's 16-byte words
  static constexpr int W = D / 64;
  u32x4_t w[W];
  __device__ __forceinline__ void load(const char* row, int c) {
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = *reinterpret_cast<const u32x4_t*>(row + 128 * k + 16 * c);
  }
  __device__ __forceinline__ float dot(const OctetRow& o) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = dot2_bf16(w[k][e], o.w[k][e], s);
    return s;
  }
};

// NS: parts of the sweep (ksplit <= NS)
template <int D, int AM, int NS>
__global__ __launch_bounds__(kThreads, 4) void seq_finish_kernel(SeqListArgs A) {
  using T = bf16_t;
  constexpr int W = D / 64, NV = 3 * NS;
  // (how much of it decides how many workgroups a compute unit holds: the notes take the scores' place when those are in registers)
  __shared__ int items_[kWaves][8][kFinishSlots];
  __shared__ __attribute__((aligned(16))) float scores_[kWaves][kFinishSlots * 64];
  static_assert(kScanList * 8 <= kFinishSlots * 64 * 4, "a wave's notes fit its scores");
  static_assert(kScanList >= 8 * kFinishSupport, "the octets' support notes and a scanned row's candidates take turns");
  const SeqGeom& g = A.a.g;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, oct = lane >> 3, c = lane & 7;
  const int hk = blockIdx.x % g.Hkv, rest = blockIdx.x / g.Hkv, wv = rest & 3, blk = A.a.nblk - 1 - (rest >> 2);
  const int id = hk * A.a.nblk + blk;
  const SeqBlock b = A.blocks[id];
  if (b.s < 0) return;
  int vote = 0;
  for (int k = 0; k < A.ksplit; ++k) vote |= A.votes[(long long)id * A.ksplit + k];
  if (vote != 0) {
    if (wv == 0 && threadIdx.x == 0) A.dense[id] = kFlagDense;
    return;
  }
  const SeqView v{b.s, b.row0, b.n, b.L};
  SeqKeys keys, vals;
  keys.init(g, v, A.a.K, hk, false, sizeof(T));
  vals.init(g, v, A.a.V, hk, true, sizeof(T));
  const int li = wave * 8 + oct;
  SeqRow row;
  row.init<true>(g, v, hk, b.r0 + wv * 32 + li, D);
  const float r = 1.0f / (g.alpha - 1.0f), a = row.a;
  const char* qrow = reinterpret_cast<const char*>(reinterpret_cast<const T*>(A.a.Q) + (long long)(v.row0 + row.t) * g.q_st + (long long)row.head * g.q_sh);
  OctetRow<D> qw;
  qw.load(qrow, c);

  // ---- what the sweep left: entry i = c + 8 u of a part is group i / 2 of half i % 2
  const GroupNumbers<8> gn(max(v.L, 1));
  float tv[NV];
  float m1 = -kInf, last = -kInf;  // (last: the largest of the parts' last places of this lane's half)
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const float* top = A.tops + (((long long)id * A.ksplit + min(k, A.ksplit - 1)) * kWaves + wv) * (kTopWords * 64) + li + 32 * (c & 1);
    const bool there = k < A.ksplit;
#pragma unroll
    for (int u = 0; u < 3; ++u) tv[3 * k + u] = there ? top[((c >> 1) + 4 * u) * 64] : -3.4e38f;
    if (there) {
      m1 = fmaxf(m1, top[kTopGroups * 64]);
      const int places = (int)top[(kTopGroups + 1) * 64];
      last = fmaxf(last, top[(places - 1) * 64]);
    }
  }
  m1 = max8(m1);
  const bool live = row.lim > 0 && m1 > -kInf;
  const float y1 = live ? a * m1 : 0.f;
  float lo = y1 - 1.0f;
  if (live && a > 1.0e-30f) {  // (entries of no key are about -3e38: a row whose a is so small that they could count keeps the bound it has)
    // Newton steps from the left on the groups' largest scores, which are scores of different keys: every iterate is a bound
    float t = lo;
#pragma unroll 1
    for (int it = 0; it < 5; ++it) {
      float f = 0.f, fp = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const float x = fmaxf(a * gn.lower(tv[k]) - t, 0.f);
        const float gx = x > 0.f ? pow_rm1<AM>(x, r) : 0.f;
        f = fmaf(gx, x, f);
        fp += gx;
      }
      f = sum8(f);
      fp = sum8(fp);
      const bool up = f > 1.0f + 1e-5f;  // (what less would add is not worth a step)
      if (__ballot(up) == 0ull) break;
      if (up) t += (f - 1.0f) * __builtin_amdgcn_rcpf(r * fp);
    }
    lo = fmaxf(lo, t - 4e-6f * fmaxf(1.0f, fabsf(t)));
  }
  const float cut = raw_cut(a, live, lo);
  if (c == 0) A.bounds[(long long)id * kBlockRows + wv * 32 + li] = make_float2(lo - y1, live ? m1 : -kInf);
  if (__builtin_amdgcn_readfirstlane(__hip_atomic_load(&A.dense[id], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) != 0)
    return;  // (others of the block's rows have given it up)

  // ---- the groups above the bound
  int* items = items_[wave][oct];
  int n = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const bool above = live && tv[k] > -3.1e38f && gn.upper(tv[k]) > cut;
    const unsigned mask = (unsigned)(__ballot(above) >> (8 * oct)) & 0xffu;
    const int place = n + (int)__popc(mask & ((1u << c) - 1u));
    if (above && place < kFinishSlots) items[place] = (int)((__float_as_uint(tv[k]) & ~gn.keep) << 1) | (c & 1);
    n += (int)__popc(mask);
  }
  const bool lost = live && max8(last > -3.1e38f && gn.upper(last) > cut ? 1.f : 0.f) > 0.f;
  const bool hard = lost || n > kFinishSlots;
  const unsigned long long hard_octets = __ballot(hard && c == 0), lost_octets = __ballot(lost && c == 0);
  int groups = c == 0 && !lost ? n : 0;  // of the wave's rows that remember all of theirs
#pragma unroll
  for (int off = 8; off < 64; off <<= 1) groups += __shfl_xor(groups, off);
  groups = __builtin_amdgcn_readfirstlane(groups);
  // Rescoring goes by the groups, the sweeps of the tiled kernel by the keys.  One row that has lost groups among rows of few is an exception and
  // looked through key by key; among rows of many it is one of several of its block.
  if (groups > SweepAgain<T>::most_groups(v.L) / 4 || (int)__popcll(hard_octets) > kHardRows || (int)__popcll(lost_octets) > 1 ||
      (lost_octets != 0ull && (groups > kScanGroups || __ballot(lost && row.lim > kScanKeys) != 0ull))) {
    if (lane == 0) A.dense[id] = kFlagWithBounds;
    return;  // (no barriers in this kernel)
  }
  __builtin_amdgcn_wave_barrier();
  if (hard) n = 0;

  // score of key `first + 8 (c / 4) + c % 4` (span 12) or `first + c` (span 8) for the octet's eight keys; the octet's row is qw_
  auto eight = [&](int first, bool strided, const OctetRow<D>& qw_) {
    OctetRow<D> kw[8];
    // (all eight within one page; keys behind the last one repeat it)
    const int jp = min(first, v.L - 1);
    const int pg = keys.page(jp);
    const char* at = keys.row_in(pg, jp);
    const uint32_t sn = (uint32_t)keys.sn;
    const int most = v.L - 1 - jp;
#pragma unroll
    for (int k = 0; k < 8; ++k) kw[k].load(at + (uint32_t)min(strided ? 8 * (k >> 2) + (k & 3) : k, most) * sn, c);
    float s[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] = kw[k].dot(qw_);
    const float d = octet_scatter_sum(s, c);
    return keys.is_hole(pg) ? -kInf : d;
  };
  // features of this lane: 8 c .. 8 c + 7 (and 64 further on), added up over value rows
  float acc[W][8];
  auto clear = [&]() {
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[k][e] = 0.f;
  };
  auto add = [&](const OctetRow<D>& vw, float p) {
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[k][e] = fmaf(p, word_elem<T>(vw.w[k], e), acc[k][e]);
  };
  // acc += the values of entries e0, e0 + step, .. < cnt of a list, four on their way at a time
  auto gather = [&](const float2* list, int e0, int step, int cnt) {
    for (int e = e0; __ballot(e < cnt) != 0ull; e += 4 * step) {
      float2 en[4];
      int pg[4];
      OctetRow<D> vw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        en[u] = e + u * step < cnt ? list[e + u * step] : make_float2(0.f, 0.f);
        pg[u] = e + u * step < cnt ? vals.page(__float_as_int(en[u].x)) : 0;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (e + u * step < cnt) vw[u].load(vals.row_in(pg[u], __float_as_int(en[u].x)), c);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (e + u * step < cnt) add(vw[u], en[u].y);
    }
  };
  auto store = [&](const SeqRow& rw) {
    char* o = reinterpret_cast<char*>(reinterpret_cast<T*>(A.a.O) + (long long)(v.row0 + rw.t) * g.o_st + (long long)rw.head * g.o_sh);
#pragma unroll
    for (int k = 0; k < W; ++k) *reinterpret_cast<u32x4_t*>(o + 128 * k + 16 * c) = Elem<T>::pack(acc[k]).v;
  };
  auto left_end = [&](int lim) { return -__builtin_amdgcn_exp2f(-(g.alpha - 1.0f) * __builtin_amdgcn_logf((float)max(lim, 1))); };

  float2* const wave_notes = reinterpret_cast<float2*>(scores_[wave]);
  float2* notes = wave_notes + oct * kFinishSupport;
  // ---- the groups' scores: slot k of this lane's row at ys[k * 64]
  float* ys = scores_[wave] + lane;
  float top = -kInf;
  int most = n;  // over the wave's rows
#pragma unroll
  for (int off = 8; off < 64; off <<= 1) most = max(most, __shfl_xor(most, off));
  most = __builtin_amdgcn_readfirstlane(most);
  auto key_of = [&](int it) { return OctetScores<QCtx<T, D>, T, D, 8>::first_key(it >> 1, it & 1) + 8 * (c >> 2) + (c & 3); };
  for (int k = 0; k < most; ++k) {
    const int it = k < n ? items[k] : 0, j = key_of(it);
    float d = eight(j - 8 * (c >> 2) - (c & 3), true, qw);
    const bool there = k < n && j < row.lim && d > -3.0e38f;  // (-inf: a hole)
    d = fmaf(row.w, (float)max(row.pos - j, 0), row.signed_dot(d));
    d = there ? d : -kInf;
    top = fmaxf(top, d);
    ys[k * 64] = d;
  }
  top = max8(top);
  const bool some = top > -kInf;
  // ---- threshold, output; SLOTS: groups held in registers (chosen per wave)
  auto finish = [&](auto slots_) {
    constexpr int SLOTS = decltype(slots_)::value;
    float y[SLOTS];
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      y[k] = k < most ? ys[k * 64] : -kInf;
      y[k] = y[k] > -kInf ? a * (y[k] - top) : -kInf;
    }
    __builtin_amdgcn_wave_barrier();
    // (the bound is nearly the threshold where every group has one key that counts)
    float blo = -1.f, bhi = left_end(row.lim), tau = fminf(fmaxf(lo - a * top - 1e-5f * fmaxf(1.f, fabsf(lo)), -1.f), bhi);
    bool done = !some;
    for (int it = 0; __ballot(!done) != 0ull && it < kMaxSolveIters; ++it) {
      RowSums sums;
      sums.clear();
#pragma unroll
      for (int k = 0; k < SLOTS; ++k) accumulate<AM>(sums, y[k] - tau, r);
      sums.s0 = sum8(sums.s0);
      sums.s1 = sum8(sums.s1);
      sums.s2 = sum8(sums.s2);
      sums.xmin = min8(sums.xmin);
      if (!done) done = solve_step<AM>(sums, r, tau, blo, bhi);
    }
    clear();
    int cnt = 0;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      const float p = some ? pow_r<AM>(fmaxf(y[k] - tau, 0.f), r) : 0.f;
      const unsigned long long all = __ballot(p > 0.f);
      if (all == 0ull) continue;
      const unsigned mask = (unsigned)(all >> (8 * oct)) & 0xffu;
      if (p > 0.f) notes[cnt + (int)__popc(mask & ((1u << c) - 1u))] = make_float2(__int_as_float(key_of(items[k])), p);
      cnt += (int)__popc(mask);
      if (__ballot(cnt > kFinishSupport - 8) != 0ull) {  // no room for another eight
        __builtin_amdgcn_wave_barrier();
        gather(notes, 0, 1, cnt);
        __builtin_amdgcn_wave_barrier();
        cnt = 0;
      }
    }
    __builtin_amdgcn_wave_barrier();
    gather(notes, 0, 1, cnt);
    if (row.valid && !hard) store(row);
  };
  if (most <= 4)
    finish(std::integral_constant<int, 4>());
  else if (most <= 12)
    finish(std::integral_constant<int, 12>());
  else
    finish(std::integral_constant<int, kFinishSlots>());

  // ---- rows that all octets look through together: their groups, or all of their keys
  for (unsigned long long rows = hard_octets; rows != 0ull; rows &= rows - 1ull) {
    const int from = __builtin_ctzll(rows);  // the octet's first lane
    const SeqRow hr = row.of_lane(from);
    const float hcut = __shfl(cut, from);
    OctetRow<D> hq;
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) hq.w[k][e] = (uint32_t)__shfl((int)qw.w[k][e], from + c);
    float2* list = wave_notes;
    int total = 0;
    float top = -kInf;
    // this lane's key j with raw product d
    auto take = [&](int j, float d) {
      const float x = fmaf(hr.w, (float)max(hr.pos - j, 0), hr.signed_dot(d));
      const bool in = j < hr.lim && d > -3.0e38f && x > hcut;
      const unsigned long long all = __ballot(in);
      const int at = total + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, 0u));
      if (in) {
        if (at < kScanList) list[at] = make_float2(__int_as_float(j), x);
        top = fmaxf(top, x);
      }
      total += (int)__popcll(all);
    };
    if (((lost_octets >> from) & 1ull) == 0ull) {
      int* wide = items_[wave][0];  // (nobody's any more)
      static_assert(24 * NS <= 8 * kFinishSlots, "a row's groups fit the octets' lists");
      int n_wide = 0;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const bool above = tv[k] > -3.1e38f && gn.upper(tv[k]) > cut;
        const unsigned mask = (unsigned)(__ballot(above) >> from) & 0xffu;
        if (above && oct == from >> 3) wide[n_wide + (int)__popc(mask & ((1u << c) - 1u))] = (int)((__float_as_uint(tv[k]) & ~gn.keep) << 1) | (c & 1);
        n_wide += (int)__popc(mask);
      }
      __builtin_amdgcn_wave_barrier();
      for (int k0 = 0; k0 < n_wide; k0 += 8) {
        const int j = key_of(wide[min(k0 + oct, n_wide - 1)]);
        const float d = eight(j - 8 * (c >> 2) - (c & 3), true, hq);
        take(k0 + oct < n_wide ? j : 0x7fffffff, d);
      }
    } else {
    constexpr int U = W == 1 ? 4 : 2;  // octets' loads under way
#pragma unroll 1
    for (int j8 = 0; j8 < hr.lim; j8 += 64 * U) {
      float d[U];
#pragma unroll
      for (int u = 0; u < U; ++u) d[u] = eight(j8 + 64 * u + 8 * oct, false, hq);
#pragma unroll
      for (int u = 0; u < U; ++u) take(j8 + 64 * u + 8 * oct + c, d[u]);
    }
    }
    if (total == 0 || total > kScanList) {  // (none: the bound came from sums in another order)
      if (lane == 0) A.dense[id] = kFlagWithBounds;
      continue;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    float2 en[kScanList / 64];
    float blo = -1.f, bhi = left_end(hr.lim), tau = -1.f;
#pragma unroll
    for (int k = 0; k < kScanList / 64; ++k) {
      en[k] = k * 64 + lane < total ? list[k * 64 + lane] : make_float2(0.f, -kInf);
      en[k].y = en[k].y > -kInf ? hr.a * (en[k].y - top) : -kInf;
    }
    bool done = false;
    for (int it = 0; !done && it < kMaxSolveIters; ++it) {
      RowSums sums;
      sums.clear();
#pragma unroll
      for (int k = 0; k < kScanList / 64; ++k) accumulate<AM>(sums, en[k].y - tau, r);
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) {
        sums.s0 += __shfl_xor(sums.s0, off);
        sums.s1 += __shfl_xor(sums.s1, off);
        sums.s2 += __shfl_xor(sums.s2, off);
        sums.xmin = fminf(sums.xmin, __shfl_xor(sums.xmin, off));
      }
      done = solve_step<AM>(sums, r, tau, blo, bhi);
    }
#pragma unroll
    for (int k = 0; k < kScanList / 64; ++k)
      if (k * 64 + lane < total) list[k * 64 + lane].y = pow_r<AM>(fmaxf(en[k].y - tau, 0.f), r);
    __builtin_amdgcn_wave_barrier();
    clear();
    gather(list, oct, 8, total);
#pragma unroll
    for (int off = 8; off < 64; off <<= 1)
#pragma unroll
      for (int k = 0; k < W; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[k][e] += __shfl_xor(acc[k][e], off);
    if (oct == 0) store(hr);
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace entmax
