// entmax_cache_plan() with its kernels on the CPU (hip/hip_runtime.h beside this file)
#include <hip/hip_runtime.h>

#include "cache_plan.hip"

extern "C" {
void emulate_begin(int order) {
  emulate::world().error[0] = 0;
  emulate::world().order = order;
}
const char* emulate_end() { return emulate::world().error; }
}
