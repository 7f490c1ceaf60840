// nf_tile.h - what the kernels that stage tiles in LDS share (nf_orthogonal.hip, nf_expert.hip).
#ifndef NF_TILE_H
#define NF_TILE_H

#include <hip/hip_runtime.h>

namespace nf {

typedef const __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;

// Until at most N of this wavefront's loads into LDS, and R of its reads of LDS, are under way.
template <int N, int R>
__device__ __forceinline__ void wait_for() {
  static_assert(N >= 0 && N < 64 && R >= 0 && R < 16, "the counters' ranges");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)" ::"n"(N), "n"(R) : "memory");
}

__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace nf
#endif  // NF_TILE_H
