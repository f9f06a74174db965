// Appending new tokens to a paged key/value cache, with the position rotation of queries and keys on the way:
//   (x, y) -> (x cos(P f_i) - y sin(P f_i), y cos(P f_i) + x sin(P f_i)) for pair i of a head's features, P the token's position.
// Every element is read and written once, so the bound is memory (24 prompts, 13300 tokens x 24 heads of 128: 32.8 us, 5.0 TB/s), and for decode steps the length of one workgroup's chain of round trips: lengths, page, rows.
//
// A thread takes units of two 16-byte chunks of a head: the two that hold the halves of the same pairs, or (interleaved pairs, and
// features that are not rotated) two neighbouring ones.  Its chunks are on their way while the angles are made: a token's
// rot / 2 angles serve all of its heads, a thread makes one of them and leaves cos and sin in LDS.
// Angles are products in 64 bits, reduced to one turn before they become 32-bit numbers (position 10^6 times a frequency of 1 has an error of
// 0.03 in 32 bits); the bits the reduced angle loses go back in through the derivative.
#include "entmax_attn.h"

#include <hip/hip_runtime.h>

#include "seq.hip.h"
#include "seq_layout.h"

using namespace entmax;

namespace {

struct AppendArgs {
  int nseq, T, Hq, Hkv;
  int lps, num_pages, max_pages, rot, interleaved;
  const int *cu, *kv_len, *table;
  const float* inv_freq;
  const char *Q, *K, *V;
  char *Qo, *Kc, *Vc;
  long long q_st, q_sh, qo_st, qo_sh, k_st, k_sh, v_st, v_sh, kc_sp, kc_sh, kc_sn, vc_sp, vc_sh, vc_sn;  // bytes
};

constexpr int kAppendThreads = kThreads;
constexpr int kAppendPer = 4;      // units of a thread under way at a time

// TB: tokens of a workgroup
template <typename T, int D, int TB>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(AppendArgs A) {
  constexpr int E = 16 / (int)sizeof(T);   // elements of a chunk
  constexpr int CH = D / E, U = CH / 2;    // chunks and units of a head
  __shared__ float2 turn[TB][64];          // (cos, sin)
  __shared__ int pos_of[TB];               // position, or -1: the token is nobody's
  __shared__ long long where_k[TB], where_v[TB];  // byte offsets of the token's place in the caches, or -1: none
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t0 = blockIdx.x * TB;
  const int heads = A.Hq + 2 * A.Hkv, per_token = heads * U;
  const int units = min(TB, A.T - t0) * per_token;
  // which rows a unit reads; first and second chunk
  auto chunks = [&](int u, bool rotated, int& c0, int& c1) {
    const int rc = A.rot / E;  // chunks that are rotated
    if (rotated && !A.interleaved && u < rc / 2) {
      c0 = u;
      c1 = u + rc / 2;
    } else {  // (units rc / 2 on: the chunks behind the rotated ones, two by two)
      c0 = 2 * u;
      c1 = 2 * u + 1;
    }
  };
  struct Place {
    int t, h, u;
  };
  auto place = [&](int x) {
    Place p;
    p.t = x / per_token;
    const int y = x - p.t * per_token;
    p.h = y / U;
    p.u = y - p.h * U;
    return p;
  };
  u32x4_t first[kAppendPer], second[kAppendPer];
  auto fetch = [&](int x0) {
#pragma unroll
    for (int k = 0; k < kAppendPer; ++k) {
      const int x = x0 + k * kAppendThreads + tid;
      if (x >= units) continue;
      const Place p = place(x);
      const long long t = t0 + p.t;
      const char* src = p.h < A.Hq ? A.Q + t * A.q_st + p.h * A.q_sh
                                   : (p.h < A.Hq + A.Hkv ? A.K + t * A.k_st + (p.h - A.Hq) * A.k_sh
                                                         : A.V + t * A.v_st + (p.h - A.Hq - A.Hkv) * A.v_sh);
      int c0, c1;
      chunks(p.u, p.h < A.Hq + A.Hkv, c0, c1);
      first[k] = *reinterpret_cast<const u32x4_t*>(src + c0 * 16);
      second[k] = *reinterpret_cast<const u32x4_t*>(src + c1 * 16);
    }
  };
  fetch(0);
  // a wave per token: its sequence, its place
  for (int t = wave; t < TB; t += kAppendThreads / 64) {
    if (t0 + t >= A.T) break;
    const int s = find_seq(A.cu, A.nseq, t0 + t, [](int c, int) { return (long long)c; });
    int pos = -1;
    long long wk = -1, wv = -1;
    if (s < A.nseq) {
      const int from = A.cu[s], to = A.cu[s + 1], L = A.kv_len[s];
      if (from >= 0 && from <= t0 + t && to > t0 + t && to <= A.T && L >= to - from && (long long)L <= ((long long)A.max_pages << A.lps)) {
        pos = L - (to - from) + (t0 + t - from);
        const int page = A.table[(long long)s * A.max_pages + (pos >> A.lps)];
        if ((unsigned)page < (unsigned)A.num_pages) {
          const int in = pos & ((1 << A.lps) - 1);
          wk = page * A.kc_sp + in * A.kc_sn;
          wv = page * A.vc_sp + in * A.vc_sn;
        }
      }
    }
    if (lane == 0) {
      pos_of[t] = pos;
      where_k[t] = wk;
      where_v[t] = wv;
    }
    if (lane < A.rot / 2 && pos >= 0) {
      const double x = (double)pos * (double)A.inv_freq[lane];
      const double turns = rint(x * 0.15915494309189535);
      // 2 pi as a double and what it leaves out
      const double rest = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, x));
      const float rf = (float)rest, dr = (float)(rest - (double)rf);
      float sn, cs;
      sincosf(rf, &sn, &cs);
      turn[t][lane] = make_float2(fmaf(-dr, sn, cs), fmaf(dr, cs, sn));
    }
  }
  __syncthreads();
  for (int x0 = 0; x0 < units; x0 += kAppendPer * kAppendThreads) {
    if (x0) fetch(x0);
#pragma unroll
    for (int k = 0; k < kAppendPer; ++k) {
      const int x = x0 + k * kAppendThreads + tid;
      if (x >= units) continue;
      const Place p = place(x);
      if (pos_of[p.t] < 0) continue;
      const bool rotated = p.h < A.Hq + A.Hkv;
      int c0, c1;
      chunks(p.u, rotated, c0, c1);
      u32x4_t ra = first[k], rb = second[k];
      if (rotated && c0 * E < A.rot) {  // (a unit is rotated wholly or, beyond a boundary of 16 features, not at all)
        float xa[E], xb[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if constexpr (sizeof(T) == 2) {
            xa[e] = __uint_as_float((e & 1) ? (ra[e >> 1] & 0xffff0000u) : (ra[e >> 1] << 16));
            xb[e] = __uint_as_float((e & 1) ? (rb[e >> 1] & 0xffff0000u) : (rb[e >> 1] << 16));
          } else {
            xa[e] = __uint_as_float(ra[e]);
            xb[e] = __uint_as_float(rb[e]);
          }
        }
        if (A.interleaved) {
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const float2 fa = turn[p.t][(c0 * E + e) / 2], fb = turn[p.t][(c1 * E + e) / 2];
            const float a0 = xa[e], a1 = xa[e + 1], b0 = xb[e], b1 = xb[e + 1];
            xa[e] = fmaf(a0, fa.x, -a1 * fa.y);
            xa[e + 1] = fmaf(a1, fa.x, a0 * fa.y);
            xb[e] = fmaf(b0, fb.x, -b1 * fb.y);
            xb[e + 1] = fmaf(b1, fb.x, b0 * fb.y);
          }
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float2 f = turn[p.t][c0 * E + e];
            const float a = xa[e], b = xb[e];
            xa[e] = fmaf(a, f.x, -b * f.y);
            xb[e] = fmaf(b, f.x, a * f.y);
          }
        }
        if constexpr (sizeof(T) == 2) {
          ra = Elem<bf16_t>::pack(xa).v;
          rb = Elem<bf16_t>::pack(xb).v;
        } else {
          ra = u32x4_t{__float_as_uint(xa[0]), __float_as_uint(xa[1]), __float_as_uint(xa[2]), __float_as_uint(xa[3])};
          rb = u32x4_t{__float_as_uint(xb[0]), __float_as_uint(xb[1]), __float_as_uint(xb[2]), __float_as_uint(xb[3])};
        }
      }
      char* dst;
      if (p.h < A.Hq) {
        dst = A.Qo + (long long)(t0 + p.t) * A.qo_st + p.h * A.qo_sh;
      } else if (p.h < A.Hq + A.Hkv) {
        if (where_k[p.t] < 0) continue;
        dst = A.Kc + where_k[p.t] + (p.h - A.Hq) * A.kc_sh;
      } else {
        if (where_v[p.t] < 0) continue;
        dst = A.Vc + where_v[p.t] + (p.h - A.Hq - A.Hkv) * A.vc_sh;
      }
      *reinterpret_cast<u32x4_t*>(dst + c0 * 16) = ra;
      *reinterpret_cast<u32x4_t*>(dst + c1 * 16) = rb;
    }
  }
}

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

template <typename T, int D>
void launch_append(const AppendArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)append_workgroups(a.T));
  if (append_tokens(a.T) == 1)
    hipLaunchKernelGGL((cache_append_kernel<T, D, 1>), grid, dim3(kAppendThreads), 0, st, a);
  else
    hipLaunchKernelGGL((cache_append_kernel<T, D, 4>), grid, dim3(kAppendThreads), 0, st, a);
}

}  // namespace

extern "C" int entmax_cache_append(const entmax_append_params* p, const void* Q, const void* K, const void* V, const int32_t* cu_seqlens,
                                   const int32_t* kv_len, const int32_t* page_table, const float* inv_freq, void* Qout, void* Kcache,
                                   void* Vcache, void* hip_stream) {
  const int rc = check_append_params(p);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->T == 0 || p->nseq == 0) return ENTMAX_ATTN_OK;
  if (!K || !V || !cu_seqlens || !kv_len || (p->max_pages > 0 && !page_table)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->num_pages > 0 && (!Kcache || !Vcache)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->Hq > 0 && (!Q || !Qout)) return ENTMAX_ATTN_INVALID_ARG;
  if (p->rot > 0 && !inv_freq) return ENTMAX_ATTN_INVALID_ARG;
  if (off16(Q) || off16(K) || off16(V) || off16(Qout) || off16(Kcache) || off16(Vcache) || off4(cu_seqlens) || off4(kv_len) ||
      off4(page_table) || off4(inv_freq))
    return ENTMAX_ATTN_MISALIGNED;
  if (!append_outputs_apart(p, Q, K, V, Qout, Kcache, Vcache)) return ENTMAX_ATTN_INVALID_ARG;
  AppendArgs a;
  a.nseq = p->nseq;
  a.T = p->T;
  a.Hq = p->Hq;
  a.Hkv = p->Hkv;
  a.lps = __builtin_ctz((unsigned)p->page_size);
  a.num_pages = p->num_pages;
  a.max_pages = p->max_pages;
  a.rot = p->rot;
  a.interleaved = p->interleaved;
  a.cu = cu_seqlens;
  a.kv_len = kv_len;
  a.table = page_table;
  a.inv_freq = inv_freq;
  a.Q = reinterpret_cast<const char*>(Q);
  a.K = reinterpret_cast<const char*>(K);
  a.V = reinterpret_cast<const char*>(V);
  a.Qo = reinterpret_cast<char*>(Qout);
  a.Kc = reinterpret_cast<char*>(Kcache);
  a.Vc = reinterpret_cast<char*>(Vcache);
  const long long es = p->dtype == ENTMAX_ATTN_BF16 ? 2 : 4;
  a.q_st = p->q_stride_t * es, a.q_sh = p->q_stride_h * es, a.qo_st = p->qo_stride_t * es, a.qo_sh = p->qo_stride_h * es;
  a.k_st = p->k_stride_t * es, a.k_sh = p->k_stride_h * es, a.v_st = p->v_stride_t * es, a.v_sh = p->v_stride_h * es;
  a.kc_sp = p->kc_stride_p * es, a.kc_sh = p->kc_stride_h * es, a.kc_sn = p->kc_stride_n * es;
  a.vc_sp = p->vc_stride_p * es, a.vc_sh = p->vc_stride_h * es, a.vc_sn = p->vc_stride_n * es;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  if (p->dtype == ENTMAX_ATTN_BF16)
    p->D == 64 ? launch_append<bf16_t, 64>(a, st) : launch_append<bf16_t, 128>(a, st);
  else
    p->D == 64 ? launch_append<float, 64>(a, st) : launch_append<float, 128>(a, st);
  return hipGetLastError() == hipSuccess ? ENTMAX_ATTN_OK : ENTMAX_ATTN_LAUNCH_FAILED;
}
