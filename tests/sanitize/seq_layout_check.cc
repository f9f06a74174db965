// The serving entry points' argument checks and workspace carving under sanitizers: random parameters; every accepted set has regions that follow one
// another in 256-byte steps and bounds that the kernels' index arithmetic rests on.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "seq_layout.h"

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

int main() {
  long accepted = 0, seen = 0;
  for (; seen < 200000; ++seen) {
    entmax_seq_params p;
    memset(&p, 0, sizeof(p));
    p.nseq = PICK(0, 1, 3, 64, 4000, 1 << 20, -1, 0x7fffffff);
    p.T = PICK(0, 1, 5, 4096, 1 << 20, 1 << 26, -3, 0x7fffffff);
    p.Hkv = PICK(1, 1, 2, 4, 8, 0, -2, 4096);
    p.Hq = p.Hkv * PICK(1, 1, 2, 3, 8, 64, 100) + (rnd() % 50 == 0);
    p.D = PICK(64, 64, 128, 128, 96, 0);
    p.dtype = PICK(0, 0, 1, 1, 2);
    p.causal = PICK(0, 1, 1, 1);
    p.path = PICK(0, 0, 0, 1);
    p.alpha = PICK(0, 1, 1, 1, 1, 1, 1) + 0.5f;
    p.delta = 1.0f;
    const bool paged = rnd() % 2;
    if (paged) {
      p.page_size = PICK(16, 32, 64, 128, 65536, 24, 8);
      p.num_pages = PICK(0, 1, 1000, 1 << 30);
      p.max_pages = PICK(0, 1, 100, 1 << 16, 0x7fffffff);
      p.max_new = PICK(0, 1, 5, 2000, 0x7fffffff);
      p.max_keys = PICK(0, 1, 33, 5000, 1 << 22, 0x7fffffff, -1);
      p.k_stride_p = p.v_stride_p = 1 << 20;
    } else {
      p.max_new = p.max_keys = PICK(0, 1, 33, 5000, 1 << 22, 0x7fffffff, -1);
    }
    p.q_stride_t = p.o_stride_t = p.k_stride_n = p.v_stride_n = PICK(128, 256, 4096, 64, 130, 1 << 24);
    p.q_stride_h = p.o_stride_h = p.k_stride_h = p.v_stride_h = PICK(128, 256, 64, 1 << 20);
    const size_t bytes = seq_workspace_bytes_of(&p);
    if (check_seq_params(&p) != ENTMAX_ATTN_OK) {
      MUST(bytes == 0);
      continue;
    }
    ++accepted;
    const SeqLayout L = make_seq_layout(&p);
    MUST(bytes == L.total && bytes >= kAlign && bytes % kAlign == 0);
    MUST(L.split || L.blocks);
    const int G = p.Hq / p.Hkv;
    // launches: fewer than 2^32 threads each
    const long long groups = seq_blocks(p.nseq, p.T, G) * p.Hkv, heads = (long long)p.nseq * p.Hkv;
    MUST(4 * groups * 256 < (1ll << 32));
    if (L.lists) {
      MUST(L.ksplit >= 1 && L.ksplit <= kSeqMostSplit);
      MUST(groups * L.ksplit * 256 < (1ll << 32));
      const size_t at[6] = {L.off_blocks, L.off_votes, L.off_dense, L.off_bounds, L.off_tops, L.split ? L.off_scores : L.total};
      for (int k = 0; k < 5; ++k) MUST(at[k] % kAlign == 0 && at[k] <= at[k + 1]);
      MUST(at[5] - at[4] >= (size_t)groups * L.ksplit * kWaves * kSeqTopWords * 64 * 4 || p.nseq == 0);
    }
    if (L.split) {
      MUST(L.rows >= 0 && L.rows <= kSplitRows && (long long)L.rows <= (long long)p.max_new * G);
      MUST(L.nblk * 32ll >= p.max_keys && L.run >= 1 && L.run <= 4);
      MUST((long long)L.splits * kWaves * L.run >= L.nblk && (long long)L.pv_splits * L.pv_keys >= p.max_keys);
      MUST(heads * L.splits * 256 < (1ll << 32) && heads * L.pv_splits * 256 < (1ll << 32) && heads * L.rows * 256 < (1ll << 32));
      const size_t at[7] = {L.off_scores, L.off_bmax, L.off_mult, L.off_found, L.off_arrived, L.off_part, L.total};
      for (int k = 0; k < 6; ++k) MUST(at[k] % kAlign == 0 && at[k] <= at[k + 1]);
    }
    entmax_append_params a;
    memset(&a, 0, sizeof(a));
    a.page_size = p.page_size;
    MUST(check_append_params(&a) != ENTMAX_ATTN_OK);
  }
  printf("ok %ld of %ld\n", accepted, seen);
  return accepted > 1000 ? 0 : 1;
}
