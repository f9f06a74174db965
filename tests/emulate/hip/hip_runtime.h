// Kernels on the CPU: enough of the runtime's names to build a kernel source for the host and run its launches, so that what depends on the order in which a
// workgroup's waves run can be tested.  Every lane is a fiber.  A wave runs until its lanes wait at a barrier or have ended, then another one does; the order of
// the waves is the caller's choice (emulate_order), so that one wave can be as far ahead of the others as the barriers allow.  Lanes meet at the operations that work across
// them; that these are reached by different lanes in different places, and waves' barriers that do not match, are recorded as errors.
#pragma once
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>

#include <functional>
#include <vector>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define asm(...)           // (only to hide values from the compiler)
#define volatile(...) ("")  // (of asm volatile: loads to LDS, which nothing here runs)

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned x = 1, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {}
};
typedef void* hipStream_t;
enum hipError_t { hipSuccess = 0 };
inline hipError_t hipGetLastError() { return hipSuccess; }

struct int2 { int x, y; };
inline int2 make_int2(int x, int y) { return int2{x, y}; }
struct float2 { float x, y; };
inline float2 make_float2(float x, float y) { return float2{x, y}; }
struct uint2 { unsigned x, y; };
struct ulonglong2 { unsigned long long x, y; };
inline ulonglong2 make_ulonglong2(unsigned long long x, unsigned long long y) { return ulonglong2{x, y}; }

namespace emulate {

constexpr int kStack = 64 * 1024;
enum State { kRun, kMeet, kBarrier, kDone };
struct Lane {
  ucontext_t at;
  State state;
  int what;                 // kMeet: the operation; kBarrier: the line
  unsigned long long value; // what it brings
};
struct Wave {
  unsigned long long values[64];
  unsigned long long active;
};
struct World {
  std::vector<Lane> lanes;
  std::vector<Wave> waves;
  std::vector<char> stacks;
  ucontext_t scheduler;
  std::function<void()> body;
  int lane = 0, threads = 0;
  int order = 0;            // 0: the first wave as far ahead as it gets, 1: the last one, 2 and above: any, by this number
  unsigned long long random = 0;
  char error[256] = "";
};
inline World& world() {
  static World w;
  return w;
}
struct Index { unsigned x, y, z; };
inline Index thread_index, block_index, block_dim, grid_dim;

inline void fail(const char* text, int a, int b) {
  if (!world().error[0]) snprintf(world().error, sizeof(world().error), "%s (%d, %d)", text, a, b);
}
inline void yield() {
  World& w = world();
  const int me = w.lane;
  swapcontext(&w.lanes[me].at, &w.scheduler);
}
// The lanes of a wave bring a value each; afterwards all of them are in values[].
inline const Wave& meet(int what, unsigned long long value) {
  World& w = world();
  Lane& l = w.lanes[w.lane];
  l.state = kMeet;
  l.what = what;
  l.value = value;
  yield();
  return w.waves[world().lane >> 6];
}
inline void barrier(int line) {
  World& w = world();
  Lane& l = w.lanes[w.lane];
  l.state = kBarrier;
  l.what = line;
  yield();
}
inline void entry() {
  World& w = world();
  w.body();
  w.lanes[w.lane].state = kDone;
  for (;;) yield();
}
// Runs wave v until its lanes wait at a barrier (true) or have ended (false)
inline bool run_wave(int v) {
  World& w = world();
  const int from = v * 64, to = from + 64 < w.threads ? from + 64 : w.threads;
  for (;;) {
    for (int i = to - 1; i >= from; --i) {  // (lane 0, which does a wave's own stores, behind the others: they run side by side in earnest)
      if (w.lanes[i].state != kRun) continue;
      w.lane = i;
      thread_index.x = (unsigned)i;
      swapcontext(&w.scheduler, &w.lanes[i].at);
    }
    int meeting = -1, waiting = -1;
    bool mixed = false;
    Wave& x = w.waves[v];
    x.active = 0;
    for (int i = from; i < to; ++i) {
      const Lane& l = w.lanes[i];
      if (l.state == kMeet) {
        mixed = mixed || (meeting >= 0 && w.lanes[meeting].what != l.what);
        meeting = i;
        x.values[i - from] = l.value;
        x.active |= 1ull << (i - from);
      } else if (l.state == kBarrier) {
        mixed = mixed || (waiting >= 0 && w.lanes[waiting].what != l.what);
        waiting = i;
      }
    }
    if (mixed) fail("lanes of a wave are in different places", v, meeting >= 0 ? w.lanes[meeting].what : w.lanes[waiting].what);
    if (meeting < 0) return waiting >= 0;
    if (waiting >= 0) fail("some lanes of a wave wait at a barrier, others at an operation across them", v, w.lanes[waiting].what);
    for (int i = from; i < to; ++i)
      if (w.lanes[i].state == kMeet) w.lanes[i].state = kRun;
  }
}
inline void run_workgroup() {
  World& w = world();
  const int n = (w.threads + 63) / 64;
  for (int i = 0; i < w.threads; ++i) {
    Lane& l = w.lanes[i];
    l.state = kRun;
    getcontext(&l.at);
    l.at.uc_stack.ss_sp = w.stacks.data() + (size_t)i * kStack;
    l.at.uc_stack.ss_size = kStack;
    l.at.uc_link = nullptr;
    makecontext(&l.at, entry, 0);
  }
  std::vector<int> at(n, 0);  // 0: may run, 1: waits, 2: ended
  for (;;) {
    int next = -1, seen = 0;
    for (int k = 0; k < n; ++k) {
      const int v = w.order == 1 ? n - 1 - k : k;
      if (at[v] != 0) continue;
      if (w.order <= 1) {
        next = v;
        break;
      }
      w.random = w.random * 6364136223846793005ull + 1442695040888963407ull;
      if ((w.random >> 33) % ++seen == 0) next = v;
    }
    if (next >= 0) {
      at[next] = run_wave(next) ? 1 : 2;
      continue;
    }
    int line = -1;
    for (int v = 0; v < n; ++v)
      if (at[v] == 1)
        for (int i = v * 64; i < w.threads && i < v * 64 + 64; ++i)
          if (w.lanes[i].state == kBarrier) {
            if (line >= 0 && line != w.lanes[i].what) fail("waves wait at different barriers", line, w.lanes[i].what);
            line = w.lanes[i].what;
            w.lanes[i].state = kRun;
          }
    if (line < 0) return;
    for (int v = 0; v < n; ++v) at[v] = at[v] == 1 ? 0 : at[v];
  }
}
template <class K, class... A>
void launch(K kernel, dim3 grid, dim3 block, A... args) {
  World& w = world();
  w.threads = (int)block.x;
  w.random = (unsigned long long)w.order;
  w.lanes.resize(w.threads);
  w.waves.resize((w.threads + 63) / 64);
  w.stacks.resize((size_t)w.threads * kStack);
  block_dim = {block.x, 1, 1};
  grid_dim = {grid.x, 1, 1};
  w.body = [=] { kernel(args...); };
  for (unsigned x = 0; x < grid.x && !w.error[0]; ++x) {
    block_index = {x, 0, 0};
    run_workgroup();
  }
}

}  // namespace emulate

#define threadIdx emulate::thread_index
#define blockIdx emulate::block_index
#define blockDim emulate::block_dim
#define gridDim emulate::grid_dim
#define __syncthreads() emulate::barrier(__LINE__)
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) emulate::launch(kernel, grid, block, __VA_ARGS__)

// ---------------------------------------------------------------- across the lanes of a wave

inline int emulate_lane() { return emulate::world().lane & 63; }
inline unsigned long long __ballot(int x) {
  const emulate::Wave& w = emulate::meet(1, x != 0);
  unsigned long long r = 0;
  for (int i = 0; i < 64; ++i)
    if ((w.active >> i & 1) && w.values[i]) r |= 1ull << i;
  return r;
}
inline int __builtin_amdgcn_readfirstlane(int x) {
  const emulate::Wave& w = emulate::meet(2, (unsigned)x);
  return (int)w.values[__builtin_ctzll(w.active)];
}
inline int __builtin_amdgcn_readlane(int x, int lane) {
  const emulate::Wave& w = emulate::meet(3, (unsigned)x);
  return (int)w.values[lane & 63];
}
template <class V>
inline V __shfl(V x, int lane) {
  unsigned bits;
  static_assert(sizeof(V) == 4, "");
  memcpy(&bits, &x, 4);
  bits = (unsigned)emulate::meet(2048, bits).values[lane & 63];
  memcpy(&x, &bits, 4);
  return x;
}
template <class V>
inline V __shfl_xor(V x, int mask) { return __shfl(x, emulate_lane() ^ mask); }
inline int __builtin_amdgcn_update_dpp(int old, int x, int ctrl, int rows, int banks, bool) {
  const int me = emulate_lane(), row = me >> 4;
  const emulate::Wave& w = emulate::meet(4 + ctrl, (unsigned)x);
  if (!(rows >> row & 1) || banks != 0xf) return old;
  int from = -1;
  if (ctrl > 0x110 && ctrl <= 0x11f)  // from lanes before in the row
    from = (me & 15) >= (ctrl & 15) ? me - (ctrl & 15) : -1;
  else if (ctrl == 0x142)             // the last lane of a row to the next one
    from = row > 0 ? 16 * row - 1 : -1;
  else if (ctrl == 0x143)             // lane 31 to the upper half
    from = row >= 2 ? 31 : -1;
  else
    emulate::fail("unknown move between lanes", ctrl, 0);
  return from >= 0 && (w.active >> from & 1) ? (int)w.values[from] : old;
}

// ---------------------------------------------------------------- numbers

template <class To, class From>
inline To emulate_bits(From x) {
  static_assert(sizeof(To) == sizeof(From), "");
  To y;
  memcpy(&y, &x, sizeof(y));
  return y;
}
inline uint32_t __float_as_uint(float x) { return emulate_bits<uint32_t>(x); }
inline float __uint_as_float(uint32_t x) { return emulate_bits<float>(x); }
inline long long __double_as_longlong(double x) { return emulate_bits<long long>(x); }
inline int __clz(int x) { return x ? __builtin_clz((unsigned)x) : 32; }
inline int __clzll(long long x) { return x ? __builtin_clzll((unsigned long long)x) : 64; }
inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
template <class A, class B>
inline auto max(A a, B b) -> decltype(a + b) { return a > b ? a : b; }
template <class A, class B>
inline auto min(A a, B b) -> decltype(a + b) { return a < b ? a : b; }
template <class V, class W>
inline V atomicAdd(V* at, W x) { const V old = *at; *at += (V)x; return old; }
template <class V>
inline V atomicMin(V* at, V x) { const V old = *at; *at = x < old ? x : old; return old; }
template <class V>
inline V atomicMax(V* at, V x) { const V old = *at; *at = x > old ? x : old; return old; }
// as the hardware's: a signaling NaN comes out as NaN, a quiet one gives way to the other number
inline bool emulate_signals(float x) { return (__float_as_uint(x) & 0x7fc00000u) == 0x7f800000u && (__float_as_uint(x) & 0x3fffffu) != 0; }
inline float emulate_max(float a, float b) { return emulate_signals(a) || emulate_signals(b) ? NAN : a != a ? b : b != b ? a : a > b ? a : b; }
inline float emulate_min(float a, float b) { return emulate_signals(a) || emulate_signals(b) ? NAN : a != a ? b : b != b ? a : a < b ? a : b; }
#define fmaxf emulate_max
#define fminf emulate_min

// (matrix products and others of the headers, which nothing here runs)
inline int __syncthreads_or(int x) {
  emulate::fail("not here", __LINE__, x);
  return x;
}
#define __builtin_amdgcn_sched_group_barrier(...)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, ...) (c)
#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, ...) (c)
#define __builtin_amdgcn_exp2f exp2f
#define __builtin_amdgcn_logf log2f

