// Sums and limits over the lanes of a wave by data-parallel moves between lanes (no LDS round trips), and over a workgroup.
#pragma once
#include <hip/hip_runtime.h>

namespace entmax {

struct Add {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a + b;
  }
};
struct Most {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a > b ? a : b;
  }
};
struct Least {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a < b ? a : b;
  }
};

// x of the lane that CTRL names; `none` in lanes that it names none for, or whose row (of 16) is not in ROWS
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V lane_move(V x, V none) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two words");
  struct Words {
    int w[sizeof(V) / 4];
  };
  Words a = __builtin_bit_cast(Words, x), b = __builtin_bit_cast(Words, none);
#pragma unroll
  for (int k = 0; k < (int)(sizeof(V) / 4); ++k) a.w[k] = __builtin_amdgcn_update_dpp(b.w[k], a.w[k], CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(V, a);
}
template <typename V>
__device__ __forceinline__ V lane_value(V x, int lane) {  // (lane: the same in all lanes)
  struct Words {
    int w[sizeof(V) / 4];
  };
  Words a = __builtin_bit_cast(Words, x);
#pragma unroll
  for (int k = 0; k < (int)(sizeof(V) / 4); ++k) a.w[k] = __builtin_amdgcn_readlane(a.w[k], lane);
  return __builtin_bit_cast(V, a);
}

// Over the lanes up to and with this one of its row of 16 lanes; then of the wave.  none: what changes nothing.  All lanes together.
template <typename V, class Op>
__device__ __forceinline__ V row_scan(V x, V none, Op op) {
  x = op(lane_move<0x111, 0xf>(x, none), x);  // from 1, 2, 4, 8 lanes before
  x = op(lane_move<0x112, 0xf>(x, none), x);
  x = op(lane_move<0x114, 0xf>(x, none), x);
  return op(lane_move<0x118, 0xf>(x, none), x);
}
template <typename V, class Op>
__device__ __forceinline__ V wave_scan(V x, V none, Op op) {
  x = row_scan(x, none, op);
  x = op(lane_move<0x142, 0xa>(x, none), x);  // the last lane of a row to the whole next one: rows 1 and 3
  return op(lane_move<0x143, 0xc>(x, none), x);  // lane 31 to rows 2 and 3
}
// The same number in all lanes
template <typename V, class Op>
__device__ __forceinline__ V wave_reduce(V x, V none, Op op) {
  return lane_value(wave_scan(x, none, op), 63);
}

// Over the workgroup of NW (at most 16) waves, in a fixed order; buf: a number per wave.  (Two barriers, so that buf may be used again at once.)
template <int NW, typename V, class Op>
__device__ __forceinline__ V block_reduce(V x, V none, V* buf, Op op) {
  static_assert(NW <= 16 && (NW & (NW - 1)) == 0, "one row of lanes");
  x = wave_reduce(x, none, op);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
  __syncthreads();
  return lane_value(row_scan(buf[threadIdx.x & (NW - 1)], none, op), NW - 1);
}
// Over the threads up to and with this one; total: over all.
template <int NW, typename V, class Op>
__device__ __forceinline__ V block_scan(V x, V none, V* buf, V& total, Op op) {
  static_assert(NW <= 16 && (NW & (NW - 1)) == 0, "one row of lanes");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  x = wave_scan(x, none, op);
  __syncthreads();
  if (lane == 63) buf[wave] = x;
  __syncthreads();
  const V w = row_scan(buf[lane & (NW - 1)], none, op);
  total = lane_value(w, NW - 1);
  return wave > 0 ? op(lane_value(w, wave - 1), x) : x;
}

}  // namespace entmax
