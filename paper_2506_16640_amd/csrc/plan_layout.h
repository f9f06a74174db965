// Host-side argument validation and workspace carving of entmax_cache_plan (include/entmax_attn.h).  Plain C++, no HIP types.
#pragma once
#include "seq_layout.h"

namespace entmax {

// One workgroup does all of a step of at most so many sequences and rows (sequences and what they got stay in LDS); larger ones take two
// launches, the sequences by one workgroup, the rows by many.  (In a graph: 2000 sequences of 2 tokens 10.5 us, 17.7 in two launches; 64 sequences of one, 4.0 and 7.7.)
constexpr int kPlanOneSeqs = 2048;
constexpr int kPlanOneRows = 4096;
constexpr int kPlanRowsPerWorkgroup = 1024;
inline bool plan_in_one(int nseq, int T) { return nseq <= kPlanOneSeqs && T <= kPlanOneRows; }

struct PlanLayout {
  size_t off_base, off_top, total;
};
inline PlanLayout make_plan_layout(const entmax_plan_params* p) {
  PlanLayout L{};
  L.off_top = 0;
  L.off_base = kAlign;
  L.total = kAlign + align_up((size_t)p->nseq * sizeof(int32_t));
  return L;
}

inline int check_plan_params(const entmax_plan_params* p) {
  if (!p) return ENTMAX_ATTN_INVALID_ARG;
  if (p->nseq < 0 || p->T < 0) return ENTMAX_ATTN_INVALID_ARG;
  const int rc = check_pages(p->page_size, p->num_pages, p->max_pages);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->nseq > (1 << 20) || p->T > (1 << 26)) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  if ((long long)p->max_pages * p->page_size > 0x7fffffffLL) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;  // (positions are 32-bit numbers)
  return ENTMAX_ATTN_OK;
}

// Whether what the plan writes is apart from the rest; lengths and the count of free pages may take the place of the old ones.
struct PlanArrays {
  const void *new_len, *release, *kv_len, *free_count;                        // read
  const void *page_table, *free_pages, *kv_len_out, *free_count_out, *cu, *slots, *positions, *sequences, *workspace;  // written
};
inline bool plan_arrays_apart(const entmax_plan_params* p, const PlanArrays& x) {
  auto row = [](const void* at, long long bytes) { return RowSet{bytes > 0 ? at : nullptr, {1, 1, 1}, {0, 0, 0}, bytes}; };
  const long long seqs = 4ll * p->nseq, rows = p->T;
  const RowSet in[4] = {row(x.new_len, seqs), row(x.release, seqs), row(x.kv_len, seqs), row(x.free_count, 4)};
  const RowSet out[9] = {row(x.page_table, seqs * p->max_pages), row(x.free_pages, 4ll * p->num_pages), row(x.kv_len_out, seqs),
                         row(x.free_count_out, 4), row(x.cu, seqs + 4), row(x.slots, 8 * rows), row(x.positions, 4 * rows),
                         row(x.sequences, 4 * rows), row(x.workspace, (long long)make_plan_layout(p).total)};
  for (int a = 0; a < 9; ++a) {
    for (int c = a + 1; c < 9; ++c)
      if (rows_meet(out[a], out[c])) return false;
    for (int c = 0; c < 4; ++c)
      if (!((a == 2 && c == 2 && x.kv_len_out == x.kv_len) || (a == 3 && c == 3 && x.free_count_out == x.free_count)) && rows_meet(out[a], in[c]))
        return false;
  }
  return true;
}

}  // namespace entmax
