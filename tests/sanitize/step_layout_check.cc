// The argument checks and workspace carving of a decode step's entry points (plan, softmax attention, sampling) under sanitizers: random parameters; every
// accepted set has regions that follow one another in 256-byte steps and bounds that the kernels' index arithmetic rests on.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "plan_layout.h"
#include "sample_layout.h"
#include "softmax_layout.h"

using namespace entmax;

static unsigned long long state = 88172645463325252ull;
static unsigned rnd() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return (unsigned)(state >> 16);
}
static int pick(const int* v, int n) { return v[rnd() % n]; }
#define PICK(...) ([]() { static const int v[] = {__VA_ARGS__}; return pick(v, (int)(sizeof(v) / sizeof(v[0]))); }())
#define MUST(x)                                              \
  if (!(x)) {                                                \
    printf("failed: %s, line %d\n", #x, __LINE__);           \
    return 1;                                                \
  }

// Pieces of `keys` keys as the kernels cut them (softmax_share): tiles of 32, at most `most` of them a piece, whole steps of tiles
static int cut(int keys, int most, int step) {
  const int tiles = (keys + 31) >> 5;
  int n = (tiles + most - 1) / most;
  if (n < 1) n = 1;
  const int each = ((tiles + n - 1) / n + step - 1) / step * step;
  if (each > 0) n = (tiles + each - 1) / each;
  return n < 1 ? 1 : n;
}

static int softmax(long& accepted) {
  entmax_seq_params p;
  memset(&p, 0, sizeof(p));
  p.nseq = PICK(0, 1, 3, 64, 200, 384, 385, 4000, 1 << 20, -1, 0x7fffffff);
  p.T = PICK(0, 1, 5, 4096, 1 << 20, 1 << 26, -3, 0x7fffffff);
  p.Hkv = PICK(1, 1, 2, 4, 8, 0, -2, 4096);
  p.Hq = p.Hkv * PICK(1, 1, 2, 3, 8, 64, 100) + (rnd() % 50 == 0);
  p.D = PICK(64, 64, 128, 128, 96, 0);
  p.dtype = PICK(0, 0, 1, 1, 2);
  p.causal = PICK(0, 1, 1, 1);
  p.path = PICK(0, 0, 0, 0, 1);
  p.alpha = PICK(1, 1, 1, 1, 1, 2);
  p.delta = 1.0f;
  p.page_size = PICK(16, 32, 64, 128, 65536, 24, 8, 0);
  p.num_pages = PICK(0, 1, 1000, 1 << 30);
  p.max_pages = PICK(0, 1, 100, 1 << 16, 0x7fffffff);
  p.max_new = PICK(0, 1, 5, 2000, 0x7fffffff);
  p.max_keys = PICK(0, 1, 33, 5000, 60000, 1 << 22, 0x7fffffff, -1);
  p.k_stride_p = p.v_stride_p = 1 << 20;
  p.q_stride_t = p.o_stride_t = p.k_stride_n = p.v_stride_n = PICK(128, 256, 4096, 64, 130, 1 << 24);
  p.q_stride_h = p.o_stride_h = p.k_stride_h = p.v_stride_h = PICK(128, 256, 64, 1 << 20);
  const size_t bytes = softmax_workspace_bytes_of(&p);
  if (check_softmax_params(&p) != ENTMAX_ATTN_OK) {
    MUST(bytes == 0);
    return 0;
  }
  ++accepted;
  const SoftmaxLayout L = make_softmax_layout(&p);
  MUST(bytes == L.total && bytes >= kAlign && bytes % kAlign == 0 && (L.split || L.blocks));
  const int G = p.Hq / p.Hkv;
  const long long groups = seq_blocks(p.nseq, p.T, G) * p.Hkv, heads = (long long)p.nseq * p.Hkv;
  size_t end = 0;
  if (L.split) {
    MUST(L.rows >= 0 && L.rows <= kSplitRows && (long long)L.rows <= (long long)p.max_new * G);
    MUST(L.most_pieces >= 1 && L.places <= heads * L.most_pieces && L.places * 256 < (1ll << 32) && heads * L.rows * 256 < (1ll << 32));
    if (!L.shared) {
      MUST(L.piece % 32 == 0 && L.splits >= 1 && L.places == heads * L.splits);
      for (int k = 0; k < 20; ++k) {
        const int keys = k == 0 ? p.max_keys : (int)(rnd() % ((unsigned)p.max_keys + 1u));
        MUST(cut(keys, L.piece / 32, 1) <= L.splits);
      }
    } else {
      // pieces of any lengths that the bounds allow: as many places as there are
      MUST(L.budget >= 1);
      static int keys[kSoftmaxSharedSeqs];
      const unsigned kind = rnd() % 4;
      long long all = 0, places = 0;
      for (int s = 0; s < p.nseq; ++s) {
        keys[s] = kind == 0 ? p.max_keys : kind == 1 ? (rnd() % 8 ? 0 : p.max_keys) : (int)(rnd() % ((unsigned)p.max_keys + 1u));
        if (kind == 3 && keys[s] > 4096) keys[s] = (int)(rnd() % 4097);
        all += keys[s] ? (keys[s] + 31) / 32 : 1;
      }
      const long long share = (all * p.Hkv + L.budget - 1) / L.budget;
      const int most = (int)(share > L.least ? share : L.least);
      for (int s = 0; s < p.nseq; ++s) {
        const int n = cut(keys[s], most, 1);
        MUST(n <= L.most_pieces);
        places += n;
      }
      MUST(places * p.Hkv <= L.places);
    }
    if (L.most_pieces > 1) {
      const size_t n = (size_t)L.places * L.rows;
      MUST(L.off_part == 0 && L.off_sums % kAlign == 0 && L.off_sums >= n * p.D * 4);
      MUST(L.off_shares % kAlign == 0 && L.off_shares >= L.off_sums + n * 8);
      end = L.off_shares + (L.shared ? (size_t)p.nseq * 8 : 0);
      MUST(end <= L.total);
    }
  }
  MUST(((L.blocks ? groups * L.tsplits : 0) + (L.split ? L.places : 0)) * 256 < (1ll << 32));
  MUST(L.tsplits >= 1 && L.tsplits <= kSoftmaxMostTiledPieces && L.tpiece % 64 == 0);
  if (L.blocks) {
    MUST(groups * L.tsplits * 256 < (1ll << 32));
    for (int k = 0; k < 20; ++k) MUST(cut(k == 0 ? p.max_keys : (int)(rnd() % ((unsigned)p.max_keys + 1u)), L.tpiece / 32, 2) <= L.tsplits);
    if (L.tsplits > 1) {
      const size_t n = (size_t)groups * L.tsplits * kBlockRows;
      MUST(L.off_tpart % kAlign == 0 && L.off_tpart >= end && L.off_tsums >= L.off_tpart + n * p.D * 4 && L.off_tsums % kAlign == 0);
      MUST(L.off_tsums + n * 8 <= L.total);
    }
  }
  return 0;
}

static int plan(long& accepted) {
  entmax_plan_params p;
  memset(&p, 0, sizeof(p));
  p.nseq = PICK(0, 1, 3, 64, 65, 2048, 2049, 1 << 20, (1 << 20) + 1, -1, 0x7fffffff);
  p.T = PICK(0, 1, 64, 4096, 4097, 1 << 26, (1 << 26) + 1, -3, 0x7fffffff);
  p.page_size = PICK(16, 32, 64, 65536, 24, 8, 0, 1 << 17, -16);
  p.num_pages = PICK(0, 1, 1000, 0x7fffffff, -1);
  p.max_pages = PICK(0, 1, 100, 1 << 15, 1 << 16, 0x7fffffff, -1);
  if (check_plan_params(&p) != ENTMAX_ATTN_OK) return 0;
  ++accepted;
  const PlanLayout L = make_plan_layout(&p);
  MUST(L.off_top + 4 <= L.off_base && L.off_base % kAlign == 0 && L.off_base + 4 * (size_t)p.nseq <= L.total && L.total % kAlign == 0);
  MUST((long long)p.max_pages * p.page_size <= 0x7fffffffll);
  // arrays one right behind the other, and each of the written ones moved onto the end of the one before
  char* const base = reinterpret_cast<char*>((size_t)1 << 44);
  const long long seqs = 4ll * p.nseq, rows = p.T;
  const long long bytes[13] = {seqs, seqs, seqs, 4, seqs * p.max_pages, 4ll * p.num_pages, seqs, 4, seqs + 4, 8 * rows, 4 * rows, 4 * rows, (long long)L.total};
  const char* at[13];
  long long o = 0;
  for (int k = 0; k < 13; ++k) {
    at[k] = base + o;
    o += bytes[k];
  }
  auto apart = [&]() { return plan_arrays_apart(&p, PlanArrays{at[0], at[1], at[2], at[3], at[4], at[5], at[6], at[7], at[8], at[9], at[10], at[11], at[12]}); };
  MUST(apart());
  for (int k = 4; k < 13; ++k)
    for (int c = 0; c < 13; ++c)
      if (c != k && bytes[k] > 0 && bytes[c] > 4) {
        const char* keep = at[k];
        at[k] = at[c] + 4;  // (never an old array as a whole)
        MUST(!apart());
        at[k] = keep;
      }
  return 0;
}

static int sample(long& accepted) {
  entmax_sample_params p;
  memset(&p, 0, sizeof(p));
  p.rows = PICK(0, 1, 3, 64, 4096, 1 << 20, (1 << 20) + 1, -1, 0x7fffffff);
  p.vocab = PICK(1, 2, 16, 50021, 131072, 200003, 1 << 21, (1 << 21) + 1, 1 << 22, (1 << 22) + 1, 0, -7, 0x7fffffff);
  p.dtype = PICK(0, 1, 0, 1, 2);
  p.stride = (long long)p.vocab + PICK(0, 0, 1, 8, 1000, -1);
  if (check_sample_params(&p) != ENTMAX_ATTN_OK) return 0;
  ++accepted;
  const SampleLayout L = make_sample_layout(&p);
  const size_t n = (size_t)p.rows * L.nslices;
  // (up to 7 elements in front of a row belong to its first slice)
  MUST((long long)L.nslices * L.slice >= (long long)p.vocab + 7 && L.nslices <= kSampleMostVocab / kSampleLargeSlice + 1 && n * 1024 < (1ull << 32));
  MUST(L.off_stat == 0 && L.off_hist >= n * kSampleStatBytes && L.off_kept >= L.off_hist + n * kSampleBins * 4);
  MUST(L.off_blocks >= L.off_kept + n * kSampleKeptBytes && L.off_cand >= L.off_blocks + n * 512);
  MUST(L.total >= L.off_cand + n * L.slice * (p.dtype == ENTMAX_ATTN_BF16 ? 4 : 8) && L.total >= kAlign);
  MUST(L.off_hist % kAlign == 0 && L.off_kept % kAlign == 0 && L.off_blocks % kAlign == 0 && L.off_cand % kAlign == 0 && L.total % kAlign == 0);
  return 0;
}

int main() {
  long accepted[3] = {0, 0, 0};
  for (int k = 0; k < 600000; ++k)
    if (softmax(accepted[0]) || (k % 8 == 0 && (plan(accepted[1]) || sample(accepted[2])))) return 1;
  for (long a : accepted) MUST(a > 1000);
  printf("ok %ld\n", accepted[0] + accepted[1] + accepted[2]);
  return 0;
}
