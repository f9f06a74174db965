// Launches of the serving attention for one (element type, head dimension); see seq_attn.hip.
#pragma once
#include "launch.hip.h"
#include "seq_decode.hip.h"
#include "seq_layout.h"
#include "seq_lists.hip.h"
#include "seq_tiled.hip.h"

namespace entmax {

struct SeqCall {
  const entmax_seq_params* p;
  const void *Q, *K, *V;
  const int32_t *cu, *kv_len, *table;
  const float *beta, *gamma, *slopes;
  void* O;
  char* ws;
  hipStream_t st;
};

// Enqueues the call for checked parameters; returns an entmax_attn_status.
template <typename T, int D>
int run_seq(const SeqCall& c);

namespace {

inline SeqGeom make_seq_geom(const SeqCall& c) {
  const entmax_seq_params* p = c.p;
  SeqGeom g;
  g.nseq = p->nseq;
  g.T = p->T;
  g.Hq = p->Hq;
  g.Hkv = p->Hkv;
  g.G = p->Hq / p->Hkv;
  g.causal = p->causal;
  g.scale_layout = p->scale_layout;
  g.logn_mode = p->logn_mode;
  g.bias_mode = p->bias_mode;
  g.alpha = p->alpha;
  g.delta = p->delta;
  g.beta = c.beta;
  g.gamma = c.gamma;
  g.slopes = c.slopes;
  g.cu = c.cu;
  g.kv_len = c.kv_len;
  g.table = c.table;
  g.lps = c.table ? __builtin_ctz((unsigned)p->page_size) : 4;
  g.num_pages = p->num_pages;
  g.max_pages = p->max_pages;
  g.max_new = p->max_new;
  g.max_keys = p->max_keys;
  g.q_st = p->q_stride_t, g.q_sh = p->q_stride_h, g.o_st = p->o_stride_t, g.o_sh = p->o_stride_h;
  g.k_sp = p->k_stride_p, g.k_sh = p->k_stride_h, g.k_sn = p->k_stride_n;
  g.v_sp = p->v_stride_p, g.v_sh = p->v_stride_h, g.v_sn = p->v_stride_n;
  return g;
}

template <typename T, int D, int AM, bool WIDE>
bool launch_seq_tiled(const SeqArgs& a_in, hipStream_t st) {
  using Cfg = SeqTiledCfg<T, D, WIDE>;
  SeqArgs a = a_in;
  // a word of marks per key tile, per more of them where that takes more than 16 KB
  a.mark_shift = 0;
  while ((a.g.max_keys / Cfg::KT >> a.mark_shift) >= 4095) ++a.mark_shift;
  a.mark_words = (a.g.max_keys / Cfg::KT >> a.mark_shift) + 1;
  const size_t smem = Cfg::lds_bytes(a.mark_words);
  constexpr auto kern = seq_tiled_kernel<T, D, AM, WIDE>;
  if (!ensure_dynamic_lds<kern>(smem)) return false;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.nblk * a.g.Hkv)), dim3(Cfg::NT), smem, st, a);
  return launch_ok();
}

template <typename T, int D, int AM>
bool launch_seq_split(const SeqDecodeArgs& a, hipStream_t st) {
  const dim3 scores((unsigned)(a.g.nseq * a.splits), (unsigned)a.g.Hkv), pv((unsigned)(a.g.nseq * a.pv_splits), (unsigned)a.g.Hkv);
  if (a.rows <= 32)
    hipLaunchKernelGGL((seq_scores_kernel<T, D, 1>), scores, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((seq_scores_kernel<T, D, 2>), scores, dim3(kThreads), 0, st, a);
  if (!launch_ok()) return false;
  // A workgroup per row, of 512 threads while three of them for every CU are as many as there are rows, else of 256; with more than 4096 rows (most of them
  // of no sequence, if some have many new tokens) a workgroup takes several in turn.
  const long long heads = (long long)a.g.nseq * a.g.Hkv;
  const int stride = (int)(heads * a.rows <= 4096 ? a.rows : (4096 / heads > 1 ? 4096 / heads : 1));
  if (heads * a.rows <= 768)
    hipLaunchKernelGGL((seq_solve_kernel<T, D, AM, 512>), dim3((unsigned)(heads * stride)), dim3(512), 0, st, a, stride);
  else
    hipLaunchKernelGGL((seq_solve_kernel<T, D, AM, 256>), dim3((unsigned)(heads * stride)), dim3(256), 0, st, a, stride);
  if (!launch_ok()) return false;
  if (a.rows <= 32)
    hipLaunchKernelGGL((seq_pv_kernel<T, D, AM, 1>), pv, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((seq_pv_kernel<T, D, AM, 2>), pv, dim3(kThreads), 0, st, a);
  return launch_ok();
}

template <int D, int AM>
bool launch_seq_lists(const SeqListArgs& a, hipStream_t st) {
  const unsigned groups = (unsigned)(a.a.nblk * a.a.g.Hkv);
  constexpr auto sweep = seq_sweep_kernel<D>;
  if (!ensure_dynamic_lds<sweep>(SeqSweepCfg<D>::kLdsBytes)) return false;
  hipLaunchKernelGGL(sweep, dim3(groups * (unsigned)a.ksplit), dim3(kThreads), SeqSweepCfg<D>::kLdsBytes, st, a);
  if (!launch_ok()) return false;
  if (a.ksplit == 1)
    hipLaunchKernelGGL((seq_finish_kernel<D, AM, 1>), dim3(4 * groups), dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((seq_finish_kernel<D, AM, 4>), dim3(4 * groups), dim3(kThreads), 0, st, a);
  return launch_ok();
}

template <typename T, int D, int AM>
bool launch_seq(const SeqArgs& a_in, const SeqListArgs& l, const SeqDecodeArgs& d, const SeqLayout& L, hipStream_t st) {
  SeqArgs a = a_in;
  if constexpr (sizeof(T) == 2) {
    if (l.ksplit > 0) {
      if (!launch_seq_lists<D, AM>(l, st)) return false;
      a.dense = l.dense;
      a.bounds = l.bounds;
      a.blocks = l.blocks;
    }
  }
  if (L.blocks) {
    const bool wide = (long long)a.nblk * a.g.Hkv < kSeqWideBelow;
    if (!(wide ? launch_seq_tiled<T, D, AM, true>(a, st) : launch_seq_tiled<T, D, AM, false>(a, st))) return false;
  }
  return !a.split || launch_seq_split<T, D, AM>(d, st);
}

}  // namespace

template <typename T, int D>
int run_seq(const SeqCall& c) {
  const entmax_seq_params* p = c.p;
  SeqLayout L = make_seq_layout(p);
  SeqArgs a;
  a.g = make_seq_geom(c);
  a.Q = c.Q;
  a.K = c.K;
  a.V = c.V;
  a.O = c.O;
  a.nblk = (int)seq_blocks(p->nseq, p->T, a.g.G);
  a.split = L.split && p->path == 0 ? 1 : 0;
  if (!a.split) L.blocks = true;
  a.dense = nullptr;
  a.bounds = nullptr;
  a.blocks = nullptr;
  SeqListArgs l;
  l.a = a;
  l.blocks = reinterpret_cast<SeqBlock*>(c.ws + L.off_blocks);
  l.bounds = reinterpret_cast<float2*>(c.ws + L.off_bounds);
  l.votes = reinterpret_cast<int*>(c.ws + L.off_votes);
  l.dense = reinterpret_cast<int*>(c.ws + L.off_dense);
  l.tops = reinterpret_cast<float*>(c.ws + L.off_tops);
  l.ksplit = L.lists && p->path == 0 ? L.ksplit : 0;
  SeqDecodeArgs d;
  d.g = a.g;
  d.Q = c.Q;
  d.K = c.K;
  d.V = c.V;
  d.O = c.O;
  d.scores = reinterpret_cast<float*>(c.ws + L.off_scores);
  d.bmax = reinterpret_cast<float*>(c.ws + L.off_bmax);
  d.mult = reinterpret_cast<float*>(c.ws + L.off_mult);
  d.found = reinterpret_cast<float2*>(c.ws + L.off_found);
  d.arrived = reinterpret_cast<int*>(c.ws + L.off_arrived);
  d.part = reinterpret_cast<float*>(c.ws + L.off_part);
  d.rows = L.rows;
  d.nblk = L.nblk;
  d.run = L.run;
  d.splits = L.splits;
  d.pv_keys = L.pv_keys;
  d.pv_splits = L.pv_splits;
  bool ok = false;
  switch (alpha_mode(p->alpha)) {
    case 1: ok = launch_seq<T, D, 1>(a, l, d, L, c.st); break;
    case 2: ok = launch_seq<T, D, 2>(a, l, d, L, c.st); break;
    case 3: ok = launch_seq<T, D, 3>(a, l, d, L, c.st); break;
    default: ok = launch_seq<T, D, 0>(a, l, d, L, c.st); break;
  }
  return ok ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // namespace entmax
