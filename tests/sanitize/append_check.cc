// The append entry point's argument checks under sanitizers: random parameters; what the kernel counts in 32 bits fits for every accepted set.
#include <stdio.h>
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
    entmax_append_params p;
    memset(&p, 0, sizeof(p));
    p.nseq = PICK(0, 1, 3, 4000, 1 << 20, -1);
    p.T = PICK(0, 1, 5, 2048, 2049, 1 << 20, (1 << 26) - 4, (1 << 26) - 3, 1 << 26, -3);
    p.Hkv = PICK(1, 2, 8, 4096, 4097, 1 << 24, 0x7fffffff, 0, -2);
    p.Hq = p.Hkv > 0 && p.Hkv < 8192 ? p.Hkv * PICK(0, 1, 2, 3) : 0;
    p.D = PICK(64, 128, 128, 96);
    p.dtype = PICK(0, 1, 1, 2);
    p.page_size = PICK(16, 64, 65536, 24);
    p.num_pages = PICK(0, 1, 1 << 30);
    p.max_pages = PICK(0, 1, 100, 1 << 15, 0x7fffffff);
    p.rot = PICK(0, 16, 64, 128, 24);
    p.q_stride_t = p.qo_stride_t = p.k_stride_t = p.v_stride_t = 1ll << 30;
    p.q_stride_h = p.qo_stride_h = p.k_stride_h = p.v_stride_h = 128;
    p.kc_stride_h = p.vc_stride_h = 1 << 23;
    p.kc_stride_p = p.vc_stride_p = 1ll << 37;
    p.kc_stride_n = p.vc_stride_n = 128;
    if (check_append_params(&p) != ENTMAX_ATTN_OK) continue;
    ++accepted;
    const long long heads = (long long)p.Hq + 2ll * p.Hkv, units = heads * (p.D * (p.dtype == ENTMAX_ATTN_BF16 ? 2 : 4) / 32);
    MUST(units * append_tokens(p.T) + 4 * kThreads < 1ll << 31);
    MUST(append_workgroups(p.T) * append_tokens(p.T) >= p.T && append_workgroups(p.T) * kThreads < 1ll << 32);
    MUST((long long)p.max_pages * p.page_size < 1ll << 31 && p.rot <= p.D);
  }
  printf("ok %ld of %ld\n", accepted, seen);
  return accepted > 1000 ? 0 : 1;
}
