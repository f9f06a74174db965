// The plan of a serving step over the paged cache: who gets pages, where the new tokens' rows begin, how long the sequences become, and each
// row's place in the cache.  With P the page size, L a sequence's keys and n its new tokens,
//     need = ceil((L + n) / P) - ceil(L / P)        pages
//     granted: the sum of need up to and with this sequence is at most the free pages (or need is 0), and the sum of the tokens of those at most T
// Both sums only grow, so those that get something are always the first of those that ask, and a sequence's first page is the sum before it: two
// scans over the sequences by one workgroup (a thread a sequence, 64-bit sums: lengths may be anything), then every row looks up its own
// sequence.  A page's first token enters it into the table.
// Bound by latency: a few dependent reads of a few KB.
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "plan_layout.h"
#include "seq.hip.h"

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

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// What the rows need to know of a sequence
struct PlanSeq {
  int row0, n, L, base;  // first row, tokens granted, keys before them, first page
};

// Sums of x over the threads up to and with this one; total: over all.  (Two barriers.)
__device__ __forceinline__ long long scan_sum(long long x, long long* buf, long long& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long y = __shfl_up(x, off);
    if (lane >= off) x += y;
  }
  __syncthreads();  // (buf is free)
  if (lane == 63) buf[wave] = x;
  __syncthreads();
  long long w = buf[lane & (kPlanWaves - 1)];  // (every wave adds up the waves' sums)
#pragma unroll
  for (int off = 1; off < kPlanWaves; off <<= 1) {
    const long long y = __shfl_up(w, off);
    if ((lane & (kPlanWaves - 1)) >= off) w += y;
  }
  total = __shfl(w, kPlanWaves - 1);
  const long long before = __shfl(w, wave > 0 ? wave - 1 : 0);
  return x + (wave > 0 ? before : 0);
}

__device__ __forceinline__ long long block_max(long long x, long long* buf) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x = max(x, __shfl_xor(x, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
  __syncthreads();
  x = buf[threadIdx.x & (kPlanWaves - 1)];
#pragma unroll
  for (int off = kPlanWaves / 2; off >= 1; off >>= 1) x = max(x, __shfl_xor(x, off));
  return x;
}

struct PlanLds {
  long long buf[kPlanWaves];
  int gone[kPlanThreads];    // sequences that give their pages back
  int count[kPlanThreads];   // how many, then how many before
};

// Pages of released sequences go on top of the free ones, in their order; returns the number of free pages after that.  Entries that are no page are
// passed over, and what would not fit the list is dropped.
__device__ int take_back(const PlanArgs& A, PlanLds& lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int top = max(0, min(A.free_count[0], A.num_pages));
  if (!A.release) return top;
  const int P1 = (1 << A.lps) - 1;
  for (int s0 = 0; s0 < A.nseq; s0 += kPlanThreads) {
    const int s = s0 + tid;
    const bool mine = s < A.nseq && A.release[s] != 0;
    long long found;
    const long long at = scan_sum(mine ? 1 : 0, lds.buf, found);
    if (mine) lds.gone[at - 1] = s;
    __syncthreads();
    const int n = (int)found;
    auto entries = [&](int i) {  // (a length that no table row holds has nothing to give back beyond it)
      const long long L = A.kv_len[lds.gone[i]];
      return L <= 0 ? 0 : (int)min((L + P1) >> A.lps, (long long)A.max_pages);
    };
    auto page = [&](int i, int e, int last) {
      const int pg = e < last ? A.table[(long long)lds.gone[i] * A.max_pages + e] : -1;
      return (unsigned)pg < (unsigned)A.num_pages ? pg : -1;
    };
    for (int i = wave; i < n; i += kPlanWaves) {
      int c = 0;
      const int last = entries(i);
      for (int e0 = 0; e0 < last; e0 += 64) c += (int)__popcll(__ballot(page(i, e0 + lane, last) >= 0));
      if (lane == 0) lds.count[i] = c;
    }
    __syncthreads();
    long long all;
    const long long upto = scan_sum(tid < n ? lds.count[tid] : 0, lds.buf, all);
    if (tid < n) lds.count[tid] = (int)min(upto - lds.count[tid], (long long)A.num_pages);
    __syncthreads();
    for (int i = wave; i < n; i += kPlanWaves) {
      long long to = (long long)top + lds.count[i];
      const int last = entries(i);
      for (int e0 = 0; e0 < last; e0 += 64) {
        const int pg = page(i, e0 + lane, last);
        const unsigned long long have = __ballot(pg >= 0);
        const long long place = to + (long long)__popcll(have & ((1ull << lane) - 1ull));
        if (pg >= 0 && place < A.num_pages) A.free_pages[place] = pg;
        to += (long long)__popcll(have);
      }
    }
    top = (int)min(top + all, (long long)A.num_pages);
    __syncthreads();  // (the lists are free)
  }
  return top;
}

// The sequences: store(s, row0, n, L, base) for each; returns the number of pages taken.  All threads of the one workgroup.
template <class F>
__device__ int plan_sequences(const PlanArgs& A, PlanLds& lds, int top, F store) {
  const long long P1 = (1 << A.lps) - 1, most = (long long)A.max_pages << A.lps;
  long long asked0 = 0, rows0 = 0, rows_got = 0, taken = 0;  // of the sequences before
  for (int s0 = 0; s0 < A.nseq; s0 += kPlanThreads) {
    const int s = s0 + (int)threadIdx.x;
    long long L = 0, n = 0, need = 0;
    const bool there = s < A.nseq;
    if (there) {
      L = A.release && A.release[s] != 0 ? 0 : A.kv_len[s];
      n = A.new_len[s];
      if (n < 0 || L < 0 || L + n > most) n = 0;
      need = n ? ((L + n + P1) >> A.lps) - ((L + P1) >> A.lps) : 0;
    }
    long long asked_all, rows_all;
    const long long asked = asked0 + scan_sum(need, lds.buf, asked_all);
    if (need > 0 && asked > top) n = 0;
    const long long upto = rows0 + scan_sum(n, lds.buf, rows_all);
    const bool fits = upto <= A.T;
    rows_got = max(rows_got, block_max(there && fits ? upto : 0, lds.buf));
    const long long before = upto - n;
    const int row0 = (int)(before <= A.T ? before : rows_got);
    if (!fits) n = 0;
    taken = max(taken, block_max(n > 0 && need > 0 ? asked : 0, lds.buf));
    if (there) store(s, row0, (int)n, (int)L, (int)min(asked - need, (long long)A.num_pages));
    asked0 += asked_all;
    rows0 += rows_all;
  }
  if (threadIdx.x == 0) A.cu[A.nseq] = (int)rows_got;
  return (int)taken;
}

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

__global__ __launch_bounds__(kPlanThreads) void plan_one_kernel(PlanArgs A) {
  __shared__ PlanLds lds;
  __shared__ int row0[kPlanOneSeqs + 1];
  __shared__ int2 at[kPlanOneSeqs];  // (keys before, first page)
  const int top = take_back(A, lds);
  const int taken = plan_sequences(A, lds, top, [&](int s, int r0, int n, int L, int base) {
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
  for (int r = threadIdx.x; r < A.T; r += kPlanThreads) {
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

__global__ __launch_bounds__(kPlanThreads) void plan_sequences_kernel(PlanArgs A) {
  __shared__ PlanLds lds;
  const int top = take_back(A, lds);
  const int taken = plan_sequences(A, lds, top, [&](int s, int r0, int n, int L, int base) {
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
    hipLaunchKernelGGL(plan_one_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
  }
  hipLaunchKernelGGL(plan_sequences_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
  if (hipGetLastError() != hipSuccess) return ENTMAX_ATTN_LAUNCH_FAILED;
  const bool rows = p->T > 0 && (slots || positions || sequences || p->max_pages > 0);
  if (rows) hipLaunchKernelGGL(plan_rows_kernel, dim3((unsigned)ceil_div(p->T, kPlanRowsPerWorkgroup)), dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}

}  // extern "C"
