// Host-side argument validation and workspace carving of the serving entry points (include/entmax_attn.h: packed
// sequences, paged cache).  Plain C++, no HIP types.
#pragma once
#include "host_layout.h"
#include "seq_overlap.h"

namespace entmax {

constexpr int kSeqMostKeys = 1 << 22;      // as for the other kernels
constexpr long long kSeqMostBlocks = 1 << 23;  // workgroups of a launch (a launch has less than 2^32 threads)

constexpr int kSeqMostHeads = 4096;        // of queries, and of keys and values: a workgroup's chunks of all heads are counted in 32 bits

inline bool power_of_two(int x) { return x > 0 && (x & (x - 1)) == 0; }

// a stride in elements: 16-byte steps, byte offsets that cannot wrap
inline int check_stride(int64_t s, int64_t es, int64_t most) {
  if (s < 0) return ENTMAX_ATTN_INVALID_ARG;
  if (s > most) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  return (s * es) % 16 != 0 ? ENTMAX_ATTN_MISALIGNED : ENTMAX_ATTN_OK;
}
constexpr int64_t kMostStride = (int64_t)1 << 40;

inline int check_heads(int32_t nseq, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype) {
  if (nseq < 0 || T < 0 || Hq < 0 || Hkv <= 0) return ENTMAX_ATTN_INVALID_ARG;
  if (Hq % Hkv != 0) return ENTMAX_ATTN_INVALID_ARG;
  if (dtype != ENTMAX_ATTN_BF16 && dtype != ENTMAX_ATTN_FP32) return ENTMAX_ATTN_INVALID_ARG;
  if (D != 64 && D != 128) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  if (Hq > kSeqMostHeads || Hkv > kSeqMostHeads || nseq > (1 << 20) || T > (1 << 26)) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  return ENTMAX_ATTN_OK;
}
inline int check_pages(int32_t page_size, int32_t num_pages, int32_t max_pages) {
  if (num_pages < 0 || max_pages < 0) return ENTMAX_ATTN_INVALID_ARG;
  if (!power_of_two(page_size) || page_size < 16 || page_size > 65536) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  return ENTMAX_ATTN_OK;
}

// groups of 128 folded rows (token, head of the group) over all sequences of a key/value head: sequence s starts at group
// cu_seqlens[s] G / 128 + s, which leaves room for every sequence's ragged last group
inline long long seq_blocks(int nseq, int T, int G) { return (long long)T * G / kBlockRows + nseq; }

inline int check_seq_params(const entmax_seq_params* p) {
  if (!p) return ENTMAX_ATTN_INVALID_ARG;
  int rc = check_heads(p->nseq, p->T, p->Hq, p->Hkv, p->D, p->dtype);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->Hq == 0) return ENTMAX_ATTN_INVALID_ARG;
  if ((p->causal | p->logn_mode | p->bias_mode | p->path) & ~1) return ENTMAX_ATTN_INVALID_ARG;
  if (p->scale_layout < 0 || p->scale_layout > 2) return ENTMAX_ATTN_INVALID_ARG;
  if (!(p->alpha > 1.0f) || !(p->alpha <= 2.0f) || !isfinite(p->delta)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->max_new < 0 || p->max_keys < 0) return ENTMAX_ATTN_INVALID_ARG;
  const bool packed = p->page_size == 0 && p->num_pages == 0 && p->max_pages == 0;
  if (packed) {
    if (p->k_stride_p != 0 || p->v_stride_p != 0 || p->max_keys != p->max_new) return ENTMAX_ATTN_INVALID_ARG;
  } else {
    rc = check_pages(p->page_size, p->num_pages, p->max_pages);
    if (rc != ENTMAX_ATTN_OK) return rc;
    if (p->max_keys > (long long)p->max_pages * p->page_size) return ENTMAX_ATTN_INVALID_ARG;
  }
  if (p->max_keys > kSeqMostKeys) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  const int64_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4;
  const int64_t strides[10] = {p->q_stride_t, p->q_stride_h, p->o_stride_t, p->o_stride_h, p->k_stride_p,
                               p->k_stride_h, p->k_stride_n, p->v_stride_p, p->v_stride_h, p->v_stride_n};
  for (int k = 0; k < 10; ++k) {
    rc = check_stride(strides[k], es, kMostStride);
    if (rc != ENTMAX_ATTN_OK) return rc;
  }
  // (offsets of a few rows inside a tile are 32-bit numbers)
  if (p->k_stride_n * es > (1 << 24) || p->v_stride_n * es > (1 << 24)) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  if (p->k_stride_n < p->D || p->v_stride_n < p->D) return ENTMAX_ATTN_INVALID_ARG;  // rows overlap
  if (p->o_stride_t < p->D || (p->Hq > 1 && p->o_stride_h < p->D)) return ENTMAX_ATTN_INVALID_ARG;
  if (seq_blocks(p->nseq, p->T, p->Hq / p->Hkv) * p->Hkv * 4 > kSeqMostBlocks) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  // (launches of the kernels that split the keys: workgroups of the value kernel, of one piece of the keys each; workgroups of rows)
  if (!packed && ((long long)p->nseq * p->Hkv * (ceil_div(p->max_keys, kWaves * 32) + 1) > kSeqMostBlocks ||
                  (long long)p->nseq * p->Hkv * 64 > kSeqMostBlocks / 2))
    return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  return ENTMAX_ATTN_OK;
}

// Tokens of an append workgroup: one while that leaves the chip room, then four, whose rows are under way together.  64 tokens x 24 heads of 128: 4.1 us
// with one, 5.7 with four; 13300 tokens of them: 36.4 us with one, 32.8 with four (5.0 TB/s read and written; a large copy reaches 5.15).
inline int append_tokens(int T) { return T <= 2048 ? 1 : 4; }
inline long long append_workgroups(int T) { return ((long long)T + append_tokens(T) - 1) / append_tokens(T); }

inline int check_append_params(const entmax_append_params* p) {
  if (!p) return ENTMAX_ATTN_INVALID_ARG;
  int rc = check_heads(p->nseq, p->T, p->Hq, p->Hkv, p->D, p->dtype);
  if (rc != ENTMAX_ATTN_OK) return rc;
  rc = check_pages(p->page_size, p->num_pages, p->max_pages);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->rot < 0 || p->rot > p->D || (p->interleaved & ~1)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->rot % 16 != 0) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  if (append_workgroups(p->T) * kThreads >= 1ll << 32) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;  // (a launch has less than 2^32 threads)
  if ((long long)p->max_pages * p->page_size > 0x7fffffffLL) return ENTMAX_ATTN_UNSUPPORTED_SHAPE;
  const int64_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4;
  const int64_t strides[14] = {p->q_stride_t, p->q_stride_h, p->qo_stride_t, p->qo_stride_h, p->k_stride_t, p->k_stride_h, p->v_stride_t,
                               p->v_stride_h, p->kc_stride_p, p->kc_stride_h, p->kc_stride_n, p->vc_stride_p, p->vc_stride_h, p->vc_stride_n};
  for (int k = 0; k < 14; ++k) {
    rc = check_stride(strides[k], es, kMostStride);
    if (rc != ENTMAX_ATTN_OK) return rc;
  }
  if (p->kc_stride_n < p->D || p->vc_stride_n < p->D) return ENTMAX_ATTN_INVALID_ARG;
  if (p->Hq > 0 && (p->qo_stride_t < p->D || (p->Hq > 1 && p->qo_stride_h < p->D))) return ENTMAX_ATTN_INVALID_ARG;
  return ENTMAX_ATTN_OK;
}

// Of an attention call with checked parameters: whether O's rows are apart from each other and from what is read.  (A block of rows may be finished twice, by two
// kernels that both read its queries; other blocks read the keys at any time.)
inline bool seq_output_apart(const entmax_seq_params* p, const void* Q, const void* K, const void* V, const void* O) {
  const int64_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4;
  const RowSet o{O, {p->T, p->Hq, 1}, {p->o_stride_t * es, p->o_stride_h * es, 0}, p->D * es};
  const RowSet q{Q, {p->T, p->Hq, 1}, {p->q_stride_t * es, p->q_stride_h * es, 0}, p->D * es};
  RowSet k{K, {p->T, p->Hkv, 1}, {p->k_stride_n * es, p->k_stride_h * es, 0}, p->D * es};
  RowSet v{V, {p->T, p->Hkv, 1}, {p->v_stride_n * es, p->v_stride_h * es, 0}, p->D * es};
  if (p->page_size != 0) {
    k = RowSet{K, {p->num_pages, p->Hkv, p->page_size}, {p->k_stride_p * es, p->k_stride_h * es, p->k_stride_n * es}, p->D * es};
    v = RowSet{V, {p->num_pages, p->Hkv, p->page_size}, {p->v_stride_p * es, p->v_stride_h * es, p->v_stride_n * es}, p->D * es};
  }
  return rows_apart(o) && !rows_meet(o, q) && !rows_meet(o, k) && !rows_meet(o, v);
}

// Of an append call with checked parameters: whether what it writes is apart in itself and from what it reads; the rotated queries may take the queries' place
// (a thread writes what it has read).
inline bool append_outputs_apart(const entmax_append_params* p, const void* Q, const void* K, const void* V, const void* Qout, const void* Kcache, const void* Vcache) {
  const int64_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4, row = p->D * es;
  auto rows = [&](const void* x, int heads, int64_t st, int64_t sh) { return RowSet{x, {p->T, heads, 1}, {st * es, sh * es, 0}, row}; };
  auto cache = [&](const void* x, int64_t sp, int64_t sh, int64_t sn) {
    return RowSet{x, {p->num_pages, p->Hkv, p->page_size}, {sp * es, sh * es, sn * es}, row};
  };
  const RowSet out[3] = {rows(Qout, p->Hq, p->qo_stride_t, p->qo_stride_h), cache(Kcache, p->kc_stride_p, p->kc_stride_h, p->kc_stride_n),
                         cache(Vcache, p->vc_stride_p, p->vc_stride_h, p->vc_stride_n)};
  const RowSet in[3] = {rows(Q, p->Hq, p->q_stride_t, p->q_stride_h), rows(K, p->Hkv, p->k_stride_t, p->k_stride_h),
                        rows(V, p->Hkv, p->v_stride_t, p->v_stride_h)};
  for (int a = 0; a < 3; ++a) {
    if (!rows_apart(out[a])) return false;
    for (int c = a + 1; c < 3; ++c)
      if (rows_meet(out[a], out[c])) return false;
    for (int c = 0; c < 3; ++c)
      if (!(a == 0 && c == 0 && same_rows(out[0], in[0])) && rows_meet(out[a], in[c])) return false;
  }
  return true;
}

// Paged sequences with at most this many folded rows (new tokens x heads of a group) go to the kernels that split the keys.
// 16 sequences of 2500 to 7000 keys, 16 query heads on 4 of 128 features: with 20 folded rows 40 us there and 74 us by blocks of 128 rows, with 64
// rows 70 us there and 85 us by blocks; with 68 rows (by blocks) 87 us.
constexpr int kSplitRows = 64;

constexpr int kSeqTopWords = 14;  // words that a lane of the sweep leaves
// Workgroups that share the keys of a group of 128 rows in the sweep of the list kernels: as many as bring the launch to three for
// every CU, while a share is not shorter than 1024 keys (and the finish kernel can hold what they leave).
constexpr int kSeqMostSplit = 4;
inline int seq_ksplit(long long groups, int max_keys) {
  int n = 1;
  while (n < kSeqMostSplit && groups * n < 768 && max_keys >= 1024 * (n + 1)) ++n;
  return n;
}

// Consecutive blocks of a wave of the score kernel: as many as leave 1024 workgroups of sequences of max_keys (fewer keep memory waiting: 4 x 4 heads
// of 32768 keys 20 us with 2048 workgroups, 17 with 1024), at most four (sequences may be much shorter: 64 x 2 heads of 200 to 8192 keys 45 us with eight,
// 24 with four).  Many rows always take four, so that they know a large score sooner and write fewer of the others.
inline int seq_run(long long heads, int nblk, int rows) {
  int n = rows > 16 ? 4 : 1;
  while (n < 4 && heads * ceil_div(nblk, kWaves * 2 * n) >= 1024) n *= 2;
  return n;
}

// The tiled kernel: below so many groups of 128 rows all waves of a compute unit go to each group, from there on small workgroups, whose starts and
// waits overlap.  Some 400 groups of 300 to 6000 keys, D 64: 182 us wide, 325 us small; about 900 of 300 to 2000 keys, D 128: 205 us wide, 189 us small.
constexpr long long kSeqWideBelow = 512;

struct SeqLayout {
  bool split;       // the call may hold such sequences
  bool blocks;      // it may hold others
  size_t off_scores;
  int rows;         // rows of a head in the score buffer
  int nblk;         // 32-key blocks of a row
  int run, splits;  // of the score kernel: blocks of a wave, workgroups of a head
  int pv_keys, pv_splits;     // of the value kernel
  bool lists;       // groups of 128 rows go through the list kernels first
  int ksplit;       // workgroups that share the keys of a group in their sweep
  size_t off_blocks, off_votes, off_dense, off_bounds, off_tops;
  size_t off_bmax, off_mult, off_found, off_arrived, off_part, total;
};

inline SeqLayout make_seq_layout(const entmax_seq_params* p) {
  SeqLayout L{};
  const int G = p->Hq / p->Hkv;
  const long long most_rows = (long long)p->max_new * G;
  L.split = p->page_size != 0 && p->max_keys > 0 && G <= kSplitRows;
  L.blocks = !L.split || most_rows > kSplitRows;
  size_t o = 0;
  L.lists = p->dtype == ENTMAX_ATTN_BF16 && L.blocks;
  if (L.lists) {
    const long long groups = seq_blocks(p->nseq, p->T, G) * p->Hkv;
    L.ksplit = seq_ksplit(groups, p->max_keys);
    L.off_blocks = o;
    o += align_up((size_t)groups * 5 * sizeof(int));
    L.off_votes = o;
    o += align_up((size_t)groups * L.ksplit * sizeof(int));
    L.off_dense = o;
    o += align_up((size_t)groups * sizeof(int));
    L.off_bounds = o;
    o += align_up((size_t)groups * kBlockRows * 2 * sizeof(float));
    L.off_tops = o;
    o += align_up((size_t)groups * L.ksplit * kWaves * kSeqTopWords * 64 * sizeof(float));
  }
  if (L.split) {
    L.off_scores = o;
    const long long heads = (long long)p->nseq * p->Hkv;
    L.rows = (int)(most_rows < kSplitRows ? most_rows : kSplitRows);
    L.nblk = ceil_div(p->max_keys, 32);
    L.run = seq_run(heads, L.nblk, L.rows);
    L.splits = ceil_div(L.nblk, kWaves * L.run);
    L.pv_keys = 512;
    L.pv_splits = ceil_div(p->max_keys, L.pv_keys);
    const size_t rows = (size_t)heads * L.rows;
    o += align_up(rows * L.nblk * 32 * sizeof(float));
    L.off_bmax = o;
    o += align_up(rows * L.nblk * sizeof(float));
    L.off_mult = o;
    o += align_up(rows * sizeof(float));
    L.off_found = o;
    o += align_up(rows * 2 * sizeof(float));
    L.off_arrived = o;
    o += align_up((size_t)heads * sizeof(int));
    L.off_part = o;
    o += align_up(rows * L.pv_splits * p->D * sizeof(float));
  }
  L.total = o < kAlign ? kAlign : o;
  return L;
}

inline size_t seq_workspace_bytes_of(const entmax_seq_params* p) {
  return check_seq_params(p) == ENTMAX_ATTN_OK ? make_seq_layout(p).total : 0;
}

}  // namespace entmax
