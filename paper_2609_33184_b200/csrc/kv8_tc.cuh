// What the tensor-core kernels that walk shares of tiles (kv8.cuh) have in common.
#pragma once
#include "kv8.cuh"
#include "tc_ptx.cuh"

namespace ss {
namespace tc {

template <int N>
__device__ __forceinline__ void bar8() {
  asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Barrier of the softmax warps that also ORs a flag over their threads.
template <int N>
__device__ __forceinline__ bool bar_or8(bool mine) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
      "bar.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)mine), "n"(N)
      : "memory");
  return any != 0;
}
// Bounded wait: one try in line, the loop out of line.  A wait that gives up (or finds that another has)
// returns like one that succeeded: what follows works on whatever is there, inside the CTA's own memory
// and its own slots, until the CTA leaves.
static __device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, volatile uint32_t* abort, uint32_t* status) {
  return *abort == 0 && mbar_wait_abortable(bar, parity, abort, status);
}
__device__ __forceinline__ void wait8(uint64_t* bar, uint32_t parity, volatile uint32_t* abort, uint32_t* status) {
  if (!mbar_try_wait(bar, parity)) wait_slow(bar, parity, abort, status);
  __syncwarp();
}

// columns [col, col + N) of the calling warp's TMEM lanes
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t* r) {
  static_assert(N == 8 || N == 16, "columns");
  if (N == 16) {
    tmem_ld16(taddr, *reinterpret_cast<uint32_t(*)[16]>(r));
  } else {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
  }
}

}  // namespace tc
}  // namespace ss
