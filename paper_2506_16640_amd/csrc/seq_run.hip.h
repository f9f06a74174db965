// Launches of the serving attention for one (element type, head dimension); see seq_attn.hip.
#pragma once
#include "launch.hip.h"
#include "seq_layout.h"
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

template <typename T, int D, int AM>
bool launch_seq_tiled(const SeqArgs& a, hipStream_t st) {
  const size_t smem = SeqTiledCfg<T, D>::lds_bytes(a.mask_words);
  constexpr auto kern = seq_tiled_kernel<T, D, AM>;
  if (!ensure_dynamic_lds<kern>(smem)) return false;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.nblk * a.g.Hkv)), dim3(kThreads), smem, st, a);
  return launch_ok();
}

}  // namespace

template <typename T, int D>
int run_seq(const SeqCall& c) {
  const entmax_seq_params* p = c.p;
  SeqArgs a;
  a.g = make_seq_geom(c);
  a.Q = c.Q;
  a.K = c.K;
  a.V = c.V;
  a.O = c.O;
  a.nblk = (int)seq_blocks(p->nseq, p->T, a.g.G);
  a.mask_words = (p->max_keys + 1023) / 1024 + 1;
  bool ok = false;
  switch (alpha_mode(p->alpha)) {
    case 1: ok = launch_seq_tiled<T, D, 1>(a, c.st); break;
    case 2: ok = launch_seq_tiled<T, D, 2>(a, c.st); break;
    case 3: ok = launch_seq_tiled<T, D, 3>(a, c.st); break;
    default: ok = launch_seq_tiled<T, D, 0>(a, c.st); break;
  }
  return ok ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // namespace entmax
