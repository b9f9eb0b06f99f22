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

// Maxima over a warp's lanes of ROWS values each, halving the rows a lane holds (of N, a power of two) at every step:
// lane's result is row lane / (32 / N)'s.  (With a redux for each of 32 rows a first tile's references took 2,000 cycles
// instead of 1,750.)
template <int N, int ROWS>
__device__ __forceinline__ float rows_max(const float2 (&x)[ROWS / 2]) {
  const int lane = threadIdx.x & 31;
  float v[N];
#pragma unroll
  for (int r = 0; r < N; ++r) v[r] = r >= ROWS ? -INFINITY : r & 1 ? x[r / 2 % (ROWS / 2)].y : x[r / 2 % (ROWS / 2)].x;
  int n = N;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    if (n > 1) {
      n /= 2;
      const bool up = lane & o;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        if (i < n) {
          const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
          v[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, send, o));
        }
      }
    } else {
      v[0] = fmaxf(v[0], __shfl_xor_sync(0xffffffffu, v[0], o));
    }
  }
  return v[0];
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

// Barrier of all threads of the cluster; orders their shared memory.
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same place in the shared memory of the cluster's CTA number `rank`.  (The loads stay between the barriers, as
// all volatile ones do, but may pass stores to other memory.)
__device__ __forceinline__ uint32_t peer_addr(const void* x, int rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(x)), "r"(rank));
  return at;
}
__device__ __forceinline__ float peer_f(const float* x, int rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer_addr(x, rank)));
  return v;
}
__device__ __forceinline__ float4 peer_f4(const float* x, int rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(peer_addr(x, rank)));
  return v;
}

// The parts of a unit and row tile that a cluster's CTAs (kCluster8) have left in their shared memory - m[N], the
// row sums of four warps [N][4], a[N][D]; or (PUSHED) in this one's, see Parts8 - to the output: each CTA joins every
// cluster-th row, in the order of the parts.  By 128 threads, four head dims each, so 4 or 8 rows side by side, and ROWS of those in flight (PARTS: most
// CTAs of the cluster): with one row a pass the 16 rows a CTA of a round's cluster took 8 us.
template <int N, int D, int PARTS, int ROWS, bool PUSHED>
__device__ __forceinline__ void cluster_join8(const Attn8Params& p, const Place8& place, const float* part_m,
                                              const float* part_l, const float* part_a) {
  Seg8 g = {};
  g.b = place.b;
  g.kvh = place.kvh;
  g.row0 = place.rt * p.rows_per_tile;
  g.nrows = min(p.rows_per_tile, p.R - g.row0);
  const int c = threadIdx.x % (D / 4) * 4, step = 128 / (D / 4) * p.cluster;
#pragma unroll 1
  for (int r0 = place.rank + threadIdx.x / (D / 4) * p.cluster; r0 < g.nrows; r0 += ROWS * step) {
    float m[ROWS][PARTS];
    float4 l[ROWS][PARTS], a[ROWS][PARTS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int r = r0 + k * step;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        l[k][i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < p.cluster && r < g.nrows) {
          if (PUSHED) {  // (r = rank + row of this CTA * parts)
            const int at = (r - (int)place.rank + i) * (D + 8);
            m[k][i] = part_m[at];
            l[k][i] = *reinterpret_cast<const float4*>(part_l + at);
            a[k][i] = *reinterpret_cast<const float4*>(part_a + at + c);
          } else {
            m[k][i] = peer_f(part_m + r, i);
            l[k][i] = peer_f4(part_l + 4 * r, i);
            a[k][i] = peer_f4(part_a + r * D + c, i);
          }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int r = r0 + k * step;
      if (r >= g.nrows) break;
      float M = -INFINITY, L = 0.f;
      float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        l[k][i].x = (l[k][i].x + l[k][i].y) + (l[k][i].z + l[k][i].w);
        if (l[k][i].x != 0.f) M = fmaxf(M, m[k][i]);  // (l = 0: an empty state, whose m and a[] may be anything)
      }
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        if (l[k][i].x == 0.f) continue;
        const float f = m[k][i] == M ? 1.f : exp2f(m[k][i] - M);
        L = fmaf(f, l[k][i].x, L);
        A.x = fmaf(f, a[k][i].x, A.x);
        A.y = fmaf(f, a[k][i].y, A.y);
        A.z = fmaf(f, a[k][i].z, A.z);
        A.w = fmaf(f, a[k][i].w, A.w);
      }
      if (c == 0) put_ml8(p, g, r, M, L);
      if (p.O) {
        const float inv = (L > 0.f || L != L) ? 1.f / L : 0.f;
        const __nv_bfloat162 lo = __floats2bfloat162_rn(A.x * inv, A.y * inv), hi = __floats2bfloat162_rn(A.z * inv, A.w * inv);
        *reinterpret_cast<uint2*>(p.O + (((int64_t)g.b * p.H_kv + g.kvh) * p.R + g.row0 + r) * D + c) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
        *reinterpret_cast<float4*>(p.part_a + (((int64_t)g.b * p.H_kv + g.kvh) * p.R_stride + g.row0 + r) * D + c) = A;
      }
    }
  }
}

// The CTA's part of its unit, for the cluster's join.  PUSH (few rows): written straight into the shared memory of the
// CTA that joins the row, in a place of its own: one barrier of the cluster and local reads, instead of two and remote
// ones (one short request, three CTAs: 5.96 -> 5.66 us, called one by one 6.8 -> 6.0).  Else written where this CTA's ring was, once that is
// done with, and read by the others.
template <int N, int D, bool PUSH>
struct Parts8 {
  static constexpr int kBlock = D + 8;  // (PUSH) floats of a row's part: m, three spare, the sums of four warps, a[]
  // (PUSH) room for the rows a CTA joins, from all parts: the most of rows(c) * c for 1 to 8 CTAs
  static constexpr int kBytes = PUSH ? 14 * kBlock * 4 : 0;
  static_assert(!PUSH || N == 8, "14 blocks");
  float* at;
  uint32_t parts, rank, inv;
  __device__ __forceinline__ Parts8(float* where, const Attn8Params& p, const Place8& place)
      : at(where), parts((uint32_t)p.cluster), rank(place.rank), inv(PUSH ? 65536u / (uint32_t)p.cluster + 1 : 0) {
    if (PUSH) {
      __syncwarp();
      asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    }
  }
  // Before the first put, by every thread of the CTA: the other CTAs have started.
  __device__ __forceinline__ void ready() const {
    if (PUSH) {
      __syncwarp();
      asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
  }
  __device__ __forceinline__ uint32_t block(uint32_t row) const {  // (PUSH) address in the CTA that joins the row
    const uint32_t k = row * inv >> 16;                            // row / parts
    return peer_addr(at, (int)(row - k * parts)) + (k * parts + rank) * (kBlock * 4);
  }
  static __device__ __forceinline__ void store(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
  }
  __device__ __forceinline__ void put_m(int row, float v) const {
    if (PUSH) store(block(row), v);
    else at[row] = v;
  }
  __device__ __forceinline__ void put_l(int row, int warp, float v) const {
    if (PUSH) store(block(row) + 16 + 4 * warp, v);
    else at[N + 4 * row + warp] = v;
  }
  __device__ __forceinline__ void put_a(int row, int c, float v) const {
    if (PUSH) store(block(row) + 32 + 4 * c, v);
    else at[5 * N + row * D + c] = v;
  }
  // A CTA without a tile, by 4 * N threads.
  __device__ __forceinline__ void put_none(int tid) const {
    if (tid < 4 * N) put_l(tid >> 2, tid & 3, 0.f);
  }
  // The join, by the whole CTA.
  __device__ __forceinline__ void end(const Attn8Params& p, const Place8& place) const {
    cluster_sync();
    if (PUSH) {
      if (threadIdx.x < 128) cluster_join8<N, D, kMostCluster8, 1, true>(p, place, at, at + 4, at + 8);
      return;
    }
    if (threadIdx.x < 128) {
      if (p.cluster <= 2) cluster_join8<N, D, 2, 4, false>(p, place, at, at + N, at + 5 * N);
      else cluster_join8<N, D, kMostCluster8, 1, false>(p, place, at, at + N, at + 5 * N);
    }
    cluster_sync();  // (nobody leaves while its state may be read)
  }
};

}  // namespace tc
}  // namespace ss
