// Host-side argument validation and workspace carving of entmax_paged_softmax_fwd (include/entmax_attn.h).  Plain C++, no HIP types.
#pragma once
#include "seq_layout.h"

namespace entmax {

// Waves of a workgroup of the kernel that splits the keys (element size, head dimension)
template <int ES, int D>
constexpr int kSoftmaxWaves = ES == 4 && D == 128 ? 2 : 4;

// Workgroups of that kernel that are on the chip at a time: two on each compute unit
constexpr int kSoftmaxSlots = 512;
// Fewest 32-key tiles of a piece.  (48 sequences of 150 to 300 keys, 2 heads of 128: 20.1 us, 22.4 with 2, 21.7 with 8.)
constexpr int kSoftmaxLeastTiles = 4;
// With so many heads of all sequences, most of which have a workgroup each in any case, only the long ones are cut.  (256
// sequences of 150 to 2000 keys, 2 heads of 128: 53 us, 70 with the rule for few; to 8000 keys: 132 and 160; to 500 keys: 27, 44 with pieces of 4 tiles.)
constexpr int kSoftmaxManyHeads = 3 * kSoftmaxSlots / 4, kSoftmaxManyLeastTiles = 16;
// With at most so many sequences their lengths decide how the keys are cut up (every wave looks at all of them), else the bound of the lengths.  (2 heads of 128, keys
// 150 to 2000: 100 sequences 29 us and 42, 256 sequences 53 and 64, 512 sequences 113 and 98.)
constexpr int kSoftmaxSharedSeqs = 384;

// softmax_tiled_piece(): a group of 128 rows is cut up along its keys where there are fewer groups than workgroups on the chip: into pieces of at least so many
// keys (bf16, fp32), until there are so many workgroups.  4 x 700 tokens against 3159 to 9130 keys, 4 x 4 heads of 128 (352 groups): 250 us, 309 whole, 269 with
// three times as many pieces.  100 tokens against 12000 keys (16 groups): 51 us, 305 whole, 58 with 8 pieces of a group at most; against 1000 keys 29 us, 42 with
// pieces of 512 keys, 27 with pieces of 128, which cost 2 x 200 tokens against 2000 keys 49 us for 44.  fp32, where a tile takes four times as long: 411 tokens of 4 x 2
// heads of 64 against themselves 26 us, 50 with pieces of 256 keys, 31 with pieces of 128; 20 x 60 tokens against 1000 keys 93 us, 84, 95.
constexpr int kSoftmaxTiledWorkgroups = 768, kSoftmaxMostTiledPieces = 32, kSoftmaxLeastTiledKeys[2] = {256, 64};

struct SoftmaxLayout {
  bool split;   // the call may hold sequences of at most kSplitRows folded rows
  bool blocks;  // it may hold others
  int rows;     // rows of a head there is room for
  bool shared;  // see softmax_share()
  int budget, least;
  int piece, splits;   // keys of a piece, pieces of a sequence, where they are not shared
  int most_pieces;     // of a sequence
  long long places;    // workgroups
  int tpiece, tsplits; // softmax_tiled_kernel: most keys of a piece, pieces of a group
  size_t off_part, off_sums, off_shares, off_tpart, off_tsums, total;
};

inline SoftmaxLayout make_softmax_layout(const entmax_seq_params* p) {
  SoftmaxLayout L{};
  const int G = p->Hq / p->Hkv;
  const long long most_rows = (long long)p->max_new * G;
  L.split = G <= kSplitRows;
  L.blocks = !L.split || most_rows > kSplitRows;
  size_t o = 0;
  if (L.split) {
    const long long heads = (long long)p->nseq * p->Hkv;
    const int tiles = p->max_keys > 0 ? ceil_div(p->max_keys, 32) : 1;
    L.rows = (int)(most_rows < kSplitRows ? most_rows : kSplitRows);
    L.shared = p->nseq <= kSoftmaxSharedSeqs;
    // (pieces are rounded up, by half a piece a head on average)
    const bool many = heads >= kSoftmaxManyHeads;
    L.budget = many ? 2 * kSoftmaxSlots : (int)(kSoftmaxSlots - heads / 2);
    L.least = many ? kSoftmaxManyLeastTiles : kSoftmaxLeastTiles;
    L.piece = kSoftmaxLeastTiles * 32;
    while (L.piece < (1 << 22) && heads * ceil_div(tiles, L.piece / 32) > 2 * kSoftmaxSlots) L.piece *= 2;
    L.splits = ceil_div(tiles, L.piece / 32);
    L.most_pieces = L.shared ? ceil_div(tiles, L.least) : L.splits;
    L.places = heads * L.most_pieces;
    // (shared: the sum of tiles / piece over the heads is at most the budget, and each of them is rounded up)
    if (L.shared && L.places > L.budget + heads) L.places = L.budget + heads;
    if (L.most_pieces > 1) {
      const size_t n = (size_t)L.places * L.rows;
      L.off_part = o;
      o += align_up(n * p->D * sizeof(float));
      L.off_sums = o;
      o += align_up(n * 2 * sizeof(float));
      L.off_shares = o;
      if (L.shared) o += align_up((size_t)p->nseq * 2 * sizeof(int));
    }
  }
  L.tsplits = 1;
  L.tpiece = 1 << 22;
  if (L.blocks) {
    const long long groups = seq_blocks(p->nseq, p->T, G) * p->Hkv;
    while (groups < kSoftmaxSlots && L.tsplits < kSoftmaxMostTiledPieces && groups * L.tsplits < kSoftmaxTiledWorkgroups &&
           p->max_keys >= kSoftmaxLeastTiledKeys[p->dtype == ENTMAX_ATTN_FP32] * (L.tsplits + 1))
      ++L.tsplits;
    if (L.tsplits > 1) {
      L.tpiece = ceil_div(ceil_div(p->max_keys, L.tsplits), 64) * 64;
      const size_t n = (size_t)groups * L.tsplits * kBlockRows;
      L.off_tpart = o;
      o += align_up(n * p->D * sizeof(float));
      L.off_tsums = o;
      o += align_up(n * 2 * sizeof(float));
    }
  }
  L.total = o < kAlign ? kAlign : o;
  return L;
}

inline int check_softmax_params(const entmax_seq_params* p) {
  if (!p || p->alpha != 1.0f || p->path != 0) return ENTMAX_ATTN_INVALID_ARG;
  entmax_seq_params q = *p;
  q.alpha = 2.0f;  // (everything else is as in the entmax attention)
  const int rc = check_seq_params(&q);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->page_size == 0) return ENTMAX_ATTN_INVALID_ARG;
  // (one launch for both kinds of sequences: fewer than 2^32 threads together)
  const SoftmaxLayout L = make_softmax_layout(p);
  const long long tiled = L.blocks ? seq_blocks(p->nseq, p->T, p->Hq / p->Hkv) * p->Hkv * L.tsplits : 0;
  return (tiled + (L.split ? L.places : 0)) * kThreads < 1ll << 32 ? ENTMAX_ATTN_OK : ENTMAX_ATTN_UNSUPPORTED_SHAPE;
}

inline size_t softmax_workspace_bytes_of(const entmax_seq_params* p) {
  return check_softmax_params(p) == ENTMAX_ATTN_OK ? make_softmax_layout(p).total : 0;
}

// Whether O and lse are apart from each other, from what is read (every workgroup may read all of it at any time) and from the workspace, and the workspace from
// tensors of floats that are read.
struct SoftmaxArrays {
  const void *Q, *K, *V, *cu, *kv_len, *table, *beta, *gamma, *slopes;  // read
  const void *O, *lse, *workspace;
};
inline bool softmax_outputs_apart(const entmax_seq_params* p, const SoftmaxArrays& x) {
  if (!seq_output_apart(p, x.Q, x.K, x.V, x.O)) return false;
  const int64_t es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4, row = p->D * es;
  auto one = [](const void* at, long long bytes) { return RowSet{bytes > 0 ? at : nullptr, {1, 1, 1}, {0, 0, 0}, bytes}; };
  const long long scales = p->scale_layout == 0 ? 0 : 4ll * p->Hq * (p->scale_layout == 1 ? 1 : p->T);
  const RowSet out[3] = {RowSet{x.O, {p->T, p->Hq, 1}, {p->o_stride_t * es, p->o_stride_h * es, 0}, row}, one(x.lse, 4ll * p->Hq * p->T),
                         one(x.workspace, (long long)make_softmax_layout(p).total)};
  const RowSet in[9] = {RowSet{x.Q, {p->T, p->Hq, 1}, {p->q_stride_t * es, p->q_stride_h * es, 0}, row},
                        RowSet{x.K, {p->num_pages, p->Hkv, p->page_size}, {p->k_stride_p * es, p->k_stride_h * es, p->k_stride_n * es}, row},
                        RowSet{x.V, {p->num_pages, p->Hkv, p->page_size}, {p->v_stride_p * es, p->v_stride_h * es, p->v_stride_n * es}, row},
                        one(x.beta, scales), one(x.gamma, scales), one(x.slopes, 4ll * p->Hq),
                        one(x.cu, 4ll * p->nseq + 4), one(x.kv_len, 4ll * p->nseq), one(x.table, 4ll * p->nseq * p->max_pages)};
  for (int a = 0; a < 3; ++a) {
    for (int c = a + 1; c < 3; ++c)
      if (rows_meet(out[a], out[c])) return false;
    for (int c = 0; c < (a == 2 ? 6 : 9); ++c)
      if (rows_meet(out[a], in[c])) return false;
  }
  return true;
}

}  // namespace entmax
