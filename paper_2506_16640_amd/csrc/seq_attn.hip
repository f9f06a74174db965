// Entry points of the serving attention: argument checks and dispatch to the (element type, head dimension) launchers.
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "seq_run.hip.h"

using namespace entmax;

namespace entmax {
extern template int run_seq<bf16_t, 64>(const SeqCall&);
extern template int run_seq<bf16_t, 128>(const SeqCall&);
extern template int run_seq<float, 64>(const SeqCall&);
extern template int run_seq<float, 128>(const SeqCall&);
}  // namespace entmax

namespace {

inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

int seq_fwd(const SeqCall& c, bool paged, size_t workspace_bytes) {
  const entmax_seq_params* p = c.p;
  const int rc = check_seq_params(p);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (paged != (p->page_size != 0)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->nseq == 0 || p->T == 0 || p->max_new == 0) return ENTMAX_ATTN_OK;
  if (!c.Q || !c.O || !c.cu || !c.ws) return ENTMAX_ATTN_INVALID_ARG;
  if (paged && (!c.kv_len || (p->max_keys > 0 && !c.table))) return ENTMAX_ATTN_INVALID_ARG;  // (no keys: nothing is looked up)
  // (a cache without pages has no keys that could be read: every page number is a hole, and holes are read from page 0)
  if (paged && p->num_pages == 0 && p->max_keys > 0) return ENTMAX_ATTN_INVALID_ARG;
  if (p->max_keys > 0 && (!c.K || !c.V)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->scale_layout != 0 && (!c.beta || !c.gamma)) return ENTMAX_ATTN_INVALID_ARG;
  if (misaligned(c.Q) || misaligned(c.K) || misaligned(c.V) || misaligned(c.O) || misaligned(c.ws)) return ENTMAX_ATTN_MISALIGNED;
  if (off4(c.cu) || off4(c.kv_len) || off4(c.table) || off4(c.beta) || off4(c.gamma) || off4(c.slopes)) return ENTMAX_ATTN_MISALIGNED;
  if (workspace_bytes < seq_workspace_bytes_of(p)) return ENTMAX_ATTN_WORKSPACE_TOO_SMALL;
  if (!seq_output_apart(p, c.Q, c.K, c.V, c.O)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->dtype == ENTMAX_ATTN_BF16) return p->D == 64 ? run_seq<bf16_t, 64>(c) : run_seq<bf16_t, 128>(c);
  return p->D == 64 ? run_seq<float, 64>(c) : run_seq<float, 128>(c);
}

}  // namespace

extern "C" {

size_t entmax_seq_workspace_bytes(const entmax_seq_params* p) { return seq_workspace_bytes_of(p); }

int entmax_paged_attn_fwd(const entmax_seq_params* p, const void* Q, const void* K, const void* V, const int32_t* cu_seqlens,
                          const int32_t* kv_len, const int32_t* page_table, const float* beta, const float* gamma,
                          const float* alibi_slopes, void* O, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return seq_fwd(SeqCall{p, Q, K, V, cu_seqlens, kv_len, page_table, beta, gamma, alibi_slopes, O, reinterpret_cast<char*>(workspace),
                         reinterpret_cast<hipStream_t>(hip_stream)},
                 true, workspace_bytes);
}

int entmax_packed_attn_fwd(const entmax_seq_params* p, const void* Q, const void* K, const void* V, const int32_t* cu_seqlens,
                           const float* beta, const float* gamma, const float* alibi_slopes, void* O, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  return seq_fwd(SeqCall{p, Q, K, V, cu_seqlens, nullptr, nullptr, beta, gamma, alibi_slopes, O, reinterpret_cast<char*>(workspace),
                         reinterpret_cast<hipStream_t>(hip_stream)},
                 false, workspace_bytes);
}

}  // extern "C"
