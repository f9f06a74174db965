// Host-side argument validation and workspace carving of entmax_sample (include/entmax_attn.h).  Plain C++, no HIP types.
#pragma once
#include "seq_layout.h"

namespace entmax {

constexpr int kSampleMostVocab = 1 << 22;   // (an index has 22 bits of a token's rank)
constexpr int kSampleBins = 512;
// Logits of a workgroup: a row is cut into slices of so many (the first one may begin up to 16 bytes in front of the row, where addresses are round)
constexpr int kSampleSmallSlice = 8192, kSampleLargeSlice = 16384;
// small ones where large ones would not give most of the chip's 512 places for workgroups something to do.  (top-p, rows of 131072: 16 of them 31 us, 38 with large ones;
// 64 of them 52 with large ones, 57 with small ones.)
inline int sample_slice(int rows, int vocab) {
  return (long long)rows * ceil_div(vocab, kSampleLargeSlice) < 384 && vocab <= kSampleMostVocab / 2 ? kSampleSmallSlice : kSampleLargeSlice;
}

constexpr int kSampleStatBytes = 16, kSampleKeptBytes = 24;  // what the kernels leave of a slice

struct SampleLayout {
  int slice, nslices;
  size_t off_stat, off_hist, off_kept, off_blocks, off_cand, total;
};
inline SampleLayout make_sample_layout(const entmax_sample_params* p) {
  SampleLayout L{};
  L.slice = sample_slice(p->rows, p->vocab);
  L.nslices = ceil_div(p->vocab + 7, L.slice);
  const size_t n = (size_t)p->rows * L.nslices;
  size_t o = 0;
  L.off_stat = o;
  o += align_up(n * kSampleStatBytes);
  L.off_hist = o;
  o += align_up(n * kSampleBins * sizeof(float));
  L.off_kept = o;
  o += align_up(n * kSampleKeptBytes);
  L.off_blocks = o;
  o += align_up(n * 64 * sizeof(double));  // (64 blocks at most)
  L.off_cand = o;
  o += align_up(n * L.slice * (p->dtype == ENTMAX_ATTN_BF16 ? 4 : 8));  // (listed tokens: all of them at worst)
  L.total = o < kAlign ? kAlign : o;
  return L;
}

inline int check_sample_params(const entmax_sample_params* p) {
  if (!p) return ENTMAX_ATTN_INVALID_ARG;
  if (p->rows < 0 || p->vocab <= 0 || p->stride < p->vocab) return ENTMAX_ATTN_INVALID_ARG;
  if (p->dtype != ENTMAX_ATTN_BF16 && p->dtype != ENTMAX_ATTN_FP32) return ENTMAX_ATTN_INVALID_ARG;
  if (p->rows > (1 << 20) || p->vocab > kSampleMostVocab || p->stride > kMostStride) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  // (a launch has less than 2^32 threads)
  if ((long long)p->rows * ceil_div(p->vocab + 7, sample_slice(p->rows, p->vocab)) * 1024 >= 1ll << 32) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  return ENTMAX_ATTN_OK;
}

// Whether what a call writes is apart in itself and from what it reads
inline bool sample_outputs_apart(const entmax_sample_params* p, const void* logits, const void* uniform, const void* temperature, const void* top_k,
                                 const void* top_p, const void* min_p, const void* token, const void* logprob, const void* workspace, size_t bytes) {
  const int64_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4;
  auto one = [](const void* at, long long n) { return RowSet{at, {1, 1, 1}, {0, 0, 0}, n}; };
  const long long n = 4ll * p->rows;
  const RowSet out[3] = {one(token, n), one(logprob, n), one(workspace, (long long)bytes)};
  const RowSet in[6] = {RowSet{logits, {p->rows, 1, 1}, {p->stride * es, 0, 0}, p->vocab * es}, one(uniform, n), one(temperature, n),
                        one(top_k, n), one(top_p, n), one(min_p, n)};
  for (int a = 0; a < 3; ++a) {
    for (int c = a + 1; c < 3; ++c)
      if (rows_meet(out[a], out[c])) return false;
    for (int c = 0; c < 6; ++c)
      if (rows_meet(out[a], in[c])) return false;
  }
  return true;
}

}  // namespace entmax
