// The plan of a serving step over the paged cache: who gets pages, where the new tokens' rows begin, how long the sequences become, and each
// row's place in the cache.  With P the page size, L a sequence's keys and n its new tokens,
//     need = ceil((L + n) / P) - ceil(L / P)        pages
//     granted: the sum of need up to and with this sequence is at most the free pages (or need is 0), and the sum of the tokens of those at most T
// Both sums only grow, so those that get something are always the first of those that ask, and a sequence's first page is the sum before it: two
// scans over the sequences by one workgroup (64-bit sums: lengths may be anything), then every row looks up its own sequence.  A page's first token enters it into
// the table.  Pages of released sequences: their table rows' entries one after the other, of which those that are pages are kept, as many at a time as the
// workgroup has loads under way.
// Bound by latency: a few dependent reads of a few KB, and scans (lanes by data-parallel moves, waves over LDS; by shuffles, and entries of released rows
// looked at by a wave for each sequence, 3000 sequences took 31 us, now 14, and 256 sequences of one token 12, now 8).  One sequence: 2.8 us with a workgroup of a
// single wave, 9.6 with 16 waves.
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "plan_layout.h"
#include "seq.hip.h"
#include "wave_ops.hip.h"

using namespace entmax;

namespace {

struct PlanArgs {
  int nseq, T, lps, num_pages, max_pages;
  const int *new_len, *release;
  const int *kv_len, *free_count;  // (may be the arrays below)
  int *table, *free_pages, *kv_out, *free_out, *cu;
  long long* slots;
  int *positions, *sequences;
  int *base, *top;  // workspace: the sequences' first pages, counted from the top of the free ones; their number after what came back
};

// What the rows need to know of a sequence
struct PlanSeq {
  int row0, n, L, base;  // first row, tokens granted, keys before them, first page
};

// A workgroup of NT threads, E sequences of each at a time
template <int NT, int E>
struct PlanTeam {
  static constexpr int NW = NT / 64, kAtOnce = NT * E;
  struct Lds {
    long long buf[NW], buf2[NW];
    int gone[kAtOnce];         // sequences that give their pages back
    long long upto[kAtOnce];   // table entries up to and with theirs
  };
  // What is read of a thread's sequences s0 + E tid ..
  struct Asked {
    int keys[E], more[E];
    bool gone[E];
    __device__ __forceinline__ void read(const PlanArgs& A, int s0) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int s = s0 + (int)threadIdx.x * E + e;
        const bool there = s < A.nseq;
        keys[e] = there ? A.kv_len[s] : 0;
        more[e] = there ? A.new_len[s] : 0;
        gone[e] = there && A.release && A.release[s] != 0;
      }
    }
  };

  // Pages of released sequences go on top of the free ones, in their order; returns the number of free pages after that.  Entries that are no page are
  // passed over, and what would not fit the list is dropped.  first: of the sequences 0 ..
  static __device__ int take_back(const PlanArgs& A, Lds& lds, const Asked& first) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int top = max(0, min(A.free_count[0], A.num_pages));
    if (!A.release) return top;
    const int P1 = (1 << A.lps) - 1;
    for (int s0 = 0; s0 < A.nseq; s0 += kAtOnce) {
      Asked x = first;
      if (s0) x.read(A, s0);
      int mine = 0;
      long long entries = 0;
      auto of = [&](int e) {  // (a length that no table row holds has nothing to give back beyond it)
        return x.gone[e] && x.keys[e] > 0 ? min(((long long)x.keys[e] + P1) >> A.lps, (long long)A.max_pages) : 0;
      };
#pragma unroll
      for (int e = 0; e < E; ++e) {
        mine += x.gone[e] ? 1 : 0;
        entries += of(e);
      }
      int found;
      long long all;
      int at = block_scan<NW>(mine, 0, reinterpret_cast<int*>(lds.buf2), found, Add()) - mine;
      if (found == 0) continue;  // (uniform)
      long long upto = block_scan<NW>(entries, 0ll, lds.buf, all, Add()) - entries;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        upto += of(e);
        if (x.gone[e]) {
          lds.gone[at] = s0 + tid * E + e;
          lds.upto[at++] = upto;
        }
      }
      __syncthreads();
      constexpr int U = 8;  // entries of a lane at a time, 64 apart
      for (long long e0 = 0; e0 < all; e0 += NT * U) {
        int pg[U], have = 0, before[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long long e = e0 + wave * 64 * U + u * 64 + lane;
          int lo = 0;  // the first sequence with upto > e
          if (e < all)
            for (int n = found; n > 1;) {
              const int half = n >> 1;
              const bool up = lds.upto[lo + half - 1] <= e;
              lo += up ? half : 0;
              n = up ? n - half : half;
            }
          pg[u] = e < all ? A.table[(long long)lds.gone[lo] * A.max_pages + (int)(e - (lo ? lds.upto[lo - 1] : 0))] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if ((unsigned)pg[u] >= (unsigned)A.num_pages) pg[u] = -1;
          const unsigned long long valid = __ballot(pg[u] >= 0);
          before[u] = have + (int)__popcll(valid & ((1ull << lane) - 1ull));
          have += (int)__popcll(valid);
        }
        int waves;
        const int to = block_scan<NW>(lane == 0 ? have : 0, 0, reinterpret_cast<int*>(lds.buf2), waves, Add());  // (up to and with this wave)
        const long long from = (long long)top + __builtin_amdgcn_readfirstlane(to) - have;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (pg[u] >= 0 && from + before[u] < A.num_pages) A.free_pages[from + before[u]] = pg[u];
        top = (int)min((long long)top + waves, (long long)A.num_pages);
      }
      __syncthreads();  // (the lists are free)
    }
    return top;
  }

  // The sequences: store(s, row0, n, L, base) for each; returns the number of pages taken.  All threads of the one workgroup.
  template <class F>
  static __device__ int sequences(const PlanArgs& A, Lds& lds, int top, const Asked& first, F store) {
    const long long P1 = (1 << A.lps) - 1, most = (long long)A.max_pages << A.lps;
    long long asked0 = 0, rows0 = 0;  // of the sequences before
    int rows_got = 0, taken = 0;
    for (int s0 = 0; s0 < A.nseq; s0 += kAtOnce) {
      Asked x = first;
      if (s0) x.read(A, s0);
      long long L[E], n[E], need[E], asked_mine = 0, asked_all;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        L[e] = x.gone[e] ? 0 : x.keys[e];
        n[e] = x.more[e];
        if (n[e] < 0 || L[e] < 0 || L[e] + n[e] > most) n[e] = 0;
        need[e] = n[e] ? ((L[e] + n[e] + P1) >> A.lps) - ((L[e] + P1) >> A.lps) : 0;
        asked_mine += need[e];
      }
      const long long asked = asked0 + block_scan<NW>(asked_mine, 0ll, lds.buf, asked_all, Add()) - asked_mine;
      long long rows_mine = 0, rows_all, upto = asked;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        upto += need[e];
        if (need[e] > 0 && upto > top) n[e] = 0;
        rows_mine += n[e];
      }
      const long long rows = rows0 + block_scan<NW>(rows_mine, 0ll, lds.buf2, rows_all, Add()) - rows_mine;
      // the last row that fits, and the last page of those that get theirs
      int fit = 0, pages = 0;
      long long r = rows;
      upto = asked;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        r += n[e];
        upto += need[e];
        if (r <= A.T) fit = (int)r;
        if (r <= A.T && n[e] > 0 && need[e] > 0) pages = (int)upto;  // (at most `top`)
      }
      const int2 best = block_most(make_int2(fit, pages), reinterpret_cast<int2*>(lds.buf));
      rows_got = max(rows_got, best.x);
      taken = max(taken, best.y);
      r = rows;
      upto = asked;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int s = s0 + (int)threadIdx.x * E + e;
        if (s < A.nseq)
          store(s, (int)(r <= A.T ? r : rows_got), r + n[e] <= A.T ? (int)n[e] : 0, (int)L[e], (int)min(upto, (long long)A.num_pages));
        r += n[e];
        upto += need[e];
      }
      asked0 += asked_all;
      rows0 += rows_all;
    }
    if (threadIdx.x == 0) A.cu[A.nseq] = rows_got;
    return taken;
  }
  static __device__ __forceinline__ int2 block_most(int2 x, int2* buf) {
    x.x = wave_reduce(x.x, 0, Most());
    x.y = wave_reduce(x.y, 0, Most());
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
    __syncthreads();
    const int2 w = buf[threadIdx.x & (NW - 1)];
    return make_int2(lane_value(row_scan(w.x, 0, Most()), NW - 1), lane_value(row_scan(w.y, 0, Most()), NW - 1));
  }
};

__device__ __forceinline__ void plan_row(const PlanArgs& A, int r, int s, const PlanSeq& q, int top) {
  const int P1 = (1 << A.lps) - 1;
  const int pos = q.L + (r - q.row0), e = pos >> A.lps;
  const int fresh = e - (int)(((long long)q.L + P1) >> A.lps);
  int pg;
  if (fresh >= 0) {
    pg = A.free_pages[top - 1 - (q.base + fresh)];
    if ((pos & P1) == 0) A.table[(long long)s * A.max_pages + e] = pg;
  } else {
    pg = A.table[(long long)s * A.max_pages + e];
  }
  if (A.slots) A.slots[r] = (unsigned)pg < (unsigned)A.num_pages ? ((long long)pg << A.lps) + (pos & P1) : -1;
  if (A.positions) A.positions[r] = pos;
  if (A.sequences) A.sequences[r] = s;
}
__device__ __forceinline__ void plan_padding(const PlanArgs& A, int r) {
  if (A.slots) A.slots[r] = -1;
  if (A.positions) A.positions[r] = -1;
  if (A.sequences) A.sequences[r] = -1;
}

template <int NT, int E>
__global__ __launch_bounds__(NT) void plan_one_kernel(PlanArgs A) {
  using Team = PlanTeam<NT, E>;
  __shared__ typename Team::Lds lds;
  __shared__ int row0[NT * E + 1];
  __shared__ int2 at[NT * E];  // (keys before, first page)
  typename Team::Asked asked;
  asked.read(A, 0);
  const int top = Team::take_back(A, lds, asked);
  const int taken = Team::sequences(A, lds, top, asked, [&](int s, int r0, int n, int L, int base) {
    row0[s] = r0;
    at[s] = make_int2(L, base);
    A.cu[s] = r0;
    A.kv_out[s] = L + n;
    if (s == A.nseq - 1) row0[A.nseq] = r0 + n;
  });
  if (threadIdx.x == 0) {
    A.free_out[0] = top - taken;
    if (A.nseq == 0) row0[0] = 0;
  }
  __syncthreads();
  const int rows = row0[A.nseq];
  for (int r = threadIdx.x; r < A.T; r += NT) {
    if (r >= rows) {
      plan_padding(A, r);
      continue;
    }
    int lo = 0, n = A.nseq;  // the last sequence with row0 <= r
    while (n > 1) {
      const int half = n >> 1;
      const bool up = row0[lo + half] <= r;
      lo += up ? half : 0;
      n = up ? n - half : half;
    }
    plan_row(A, r, lo, PlanSeq{row0[lo], 0, at[lo].x, at[lo].y}, top);
  }
}

__global__ __launch_bounds__(1024) void plan_sequences_kernel(PlanArgs A) {
  using Team = PlanTeam<1024, 4>;
  __shared__ typename Team::Lds lds;
  typename Team::Asked asked;
  asked.read(A, 0);
  const int top = Team::take_back(A, lds, asked);
  const int taken = Team::sequences(A, lds, top, asked, [&](int s, int r0, int n, int L, int base) {
    A.cu[s] = r0;
    A.kv_out[s] = L + n;
    A.base[s] = base;
  });
  if (threadIdx.x == 0) {
    A.free_out[0] = top - taken;
    A.top[0] = top;
  }
}

__global__ __launch_bounds__(kThreads) void plan_rows_kernel(PlanArgs A) {
  const int r0 = blockIdx.x * kPlanRowsPerWorkgroup, r1 = min(r0 + kPlanRowsPerWorkgroup, A.T);
  const int rows = A.nseq ? A.cu[A.nseq] : 0, top = A.top[0];
  auto same = [](int c, int) { return (long long)c; };
  int first = 0, last = 0;
  if (r0 < rows) {
    first = find_seq(A.cu, A.nseq, r0, same);
    last = find_seq(A.cu, A.nseq, min(r1, rows) - 1, same);
  }
  for (int r = r0 + (int)threadIdx.x; r < r1; r += kThreads) {
    if (r >= rows) {
      plan_padding(A, r);
      continue;
    }
    int lo = first, n = last - first + 1;
    while (n > 1) {
      const int half = n >> 1;
      const bool up = A.cu[lo + half] <= r;
      lo += up ? half : 0;
      n = up ? n - half : half;
    }
    const int c0 = A.cu[lo], c1 = A.cu[lo + 1];
    plan_row(A, r, lo, PlanSeq{c0, c1 - c0, A.kv_out[lo] - (c1 - c0), A.base[lo]}, top);
  }
}

inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace

extern "C" {

size_t entmax_plan_workspace_bytes(const entmax_plan_params* p) {
  return check_plan_params(p) == ENTMAX_ATTN_OK ? make_plan_layout(p).total : 0;
}

int entmax_cache_plan(const entmax_plan_params* p, const int32_t* new_len, const int32_t* release, const int32_t* kv_len,
                      const int32_t* free_count, int32_t* page_table, int32_t* free_pages, int32_t* kv_len_out, int32_t* free_count_out,
                      int32_t* cu_seqlens, int64_t* slots, int32_t* positions, int32_t* sequences, void* workspace, size_t workspace_bytes,
                      void* hip_stream) {
  const int rc = check_plan_params(p);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!free_count || !free_count_out || !cu_seqlens || !workspace) return ENTMAX_ATTN_INVALID_ARG;
  if (p->nseq > 0 && (!new_len || !kv_len || !kv_len_out || (p->max_pages > 0 && !page_table))) return ENTMAX_ATTN_INVALID_ARG;
  if (p->num_pages > 0 && !free_pages) return ENTMAX_ATTN_INVALID_ARG;
  if (off4(new_len) || off4(release) || off4(kv_len) || off4(free_count) || off4(page_table) || off4(free_pages) || off4(kv_len_out) ||
      off4(free_count_out) || off4(cu_seqlens) || (reinterpret_cast<uintptr_t>(slots) & 7u) != 0 || off4(positions) || off4(sequences) ||
      (reinterpret_cast<uintptr_t>(workspace) & 15u) != 0)
    return ENTMAX_ATTN_MISALIGNED;
  const PlanLayout L = make_plan_layout(p);
  if (workspace_bytes < L.total) return ENTMAX_ATTN_WORKSPACE_TOO_SMALL;
  if (!plan_arrays_apart(p, PlanArrays{new_len, release, kv_len, free_count, page_table, free_pages, kv_len_out, free_count_out, cu_seqlens,
                                       slots, positions, sequences, workspace}))
    return ENTMAX_ATTN_INVALID_ARG;
  PlanArgs a;
  a.nseq = p->nseq;
  a.T = p->T;
  a.lps = __builtin_ctz((unsigned)p->page_size);
  a.num_pages = p->num_pages;
  a.max_pages = p->max_pages;
  a.new_len = new_len;
  a.release = release;
  a.kv_len = kv_len;
  a.free_count = free_count;
  a.table = page_table;
  a.free_pages = free_pages;
  a.kv_out = kv_len_out;
  a.free_out = free_count_out;
  a.cu = cu_seqlens;
  a.slots = reinterpret_cast<long long*>(slots);
  a.positions = positions;
  a.sequences = sequences;
  a.base = reinterpret_cast<int*>(reinterpret_cast<char*>(workspace) + L.off_base);
  a.top = reinterpret_cast<int*>(reinterpret_cast<char*>(workspace) + L.off_top);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  if (plan_in_one(p->nseq, p->T)) {
    // (the smallest workgroup with a thread for each sequence and row)
    if (p->nseq <= 64 && p->T <= 64)
      hipLaunchKernelGGL((plan_one_kernel<64, 1>), dim3(1), dim3(64), 0, st, a);
    else if (p->nseq <= 256 && p->T <= 256)
      hipLaunchKernelGGL((plan_one_kernel<256, 1>), dim3(1), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((plan_one_kernel<1024, kPlanOneSeqs / 1024>), dim3(1), dim3(1024), 0, st, a);
    return hipGetLastError() == hipSuccess ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
  }
  hipLaunchKernelGGL(plan_sequences_kernel, dim3(1), dim3(1024), 0, st, a);
  if (hipGetLastError() != hipSuccess) return ENTMAX_ATTN_LAUNCH_FAILED;
  const bool rows = p->T > 0 && (slots || positions || sequences || p->max_pages > 0);
  if (rows) hipLaunchKernelGGL(plan_rows_kernel, dim3((unsigned)ceil_div(p->T, kPlanRowsPerWorkgroup)), dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // extern "C"
