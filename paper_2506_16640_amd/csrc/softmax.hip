// Entry point of the softmax attention over a paged cache: argument checks and dispatch to the (element type, head dimension) launchers.
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "softmax.hip.h"

using namespace entmax;

namespace entmax {
extern template int run_softmax<bf16_t, 64>(const SoftmaxCall&);
extern template int run_softmax<bf16_t, 128>(const SoftmaxCall&);
extern template int run_softmax<float, 64>(const SoftmaxCall&);
extern template int run_softmax<float, 128>(const SoftmaxCall&);
}  // namespace entmax

namespace {
inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
}  // namespace

extern "C" {

size_t entmax_softmax_workspace_bytes(const entmax_seq_params* p) { return softmax_workspace_bytes_of(p); }

int entmax_paged_softmax_fwd(const entmax_seq_params* p, float cap, const void* Q, const void* K, const void* V, const int32_t* cu_seqlens,
                             const int32_t* kv_len, const int32_t* page_table, const float* beta, const float* gamma,
                             const float* alibi_slopes, void* O, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_softmax_params(p);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!(cap >= 0.f) || !isfinite(cap)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->nseq == 0 || p->T == 0 || p->max_new == 0) return ENTMAX_ATTN_OK;
  if (!Q || !O || !cu_seqlens || !kv_len || !workspace) return ENTMAX_ATTN_INVALID_ARG;
  // (as in the entmax attention: no keys, nothing is looked up; a cache without pages has none that could be read)
  if (p->max_keys > 0 && (!page_table || !K || !V || p->num_pages == 0)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->scale_layout != 0 && (!beta || !gamma)) return ENTMAX_ATTN_INVALID_ARG;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || misaligned(workspace)) return ENTMAX_ATTN_MISALIGNED;
  if (off4(cu_seqlens) || off4(kv_len) || off4(page_table) || off4(beta) || off4(gamma) || off4(alibi_slopes) || off4(lse))
    return ENTMAX_ATTN_MISALIGNED;
  if (workspace_bytes < softmax_workspace_bytes_of(p)) return ENTMAX_ATTN_WORKSPACE_TOO_SMALL;
  if (!softmax_outputs_apart(p, SoftmaxArrays{Q, K, V, cu_seqlens, kv_len, page_table, beta, gamma, alibi_slopes, O, lse, workspace})) return ENTMAX_ATTN_INVALID_ARG;
  const SoftmaxCall c{p, cap, Q, K, V, cu_seqlens, kv_len, page_table, beta, gamma, alibi_slopes, O, lse, reinterpret_cast<char*>(workspace),
                      reinterpret_cast<hipStream_t>(hip_stream)};
  if (p->dtype == ENTMAX_ATTN_BF16) return p->D == 64 ? run_softmax<bf16_t, 64>(c) : run_softmax<bf16_t, 128>(c);
  return p->D == 64 ? run_softmax<float, 64>(c) : run_softmax<float, 128>(c);
}

}  // extern "C"
