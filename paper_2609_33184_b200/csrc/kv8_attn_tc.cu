// Attention over the 8-bit KV cache on the tensor cores: the codes go from HBM to the MMA as they
// are, nothing dequantises them.
//
//   S^T = K Q^T    M = 128 keys of the tile, N = rows, K = d         (d / 32 steps, e4m3 x e4m3)
//   O^T = V^T P^T  M = 128 head dims,        N = rows, K = 128 keys  (4 steps, e4m3 x e5m2)
//
// as in the bf16 kernel with the keys on M; tcgen05.mma kind::f8f6f4 takes both operands in 8 bits, so
// Q and P are split into terms of 8 bits that stand side by side on the N axis (tensor work is not
// what bounds this kernel: an MMA reads its 4 KB of A in 32 cycles and needs fewer for the maths):
//  * Q row * 2^-eq (maximum in [128, 256)) = hi + lo / 16, both e4m3.  bf16 has 8 significant bits
//    and a term holds 4, so the split is exact down to 2^-14 of the row's maximum, off by at most
//    2^-22 of it below.  The score is (S_hi + S_lo / 16) * 2^eq * 2^ek * scale: all factors powers of two
//    but the caller's, the sums in fp32.
//  * weights.  x = s2 + ev - M + 7 with s2 the score in base 2, ev the key's value exponent, M the row's
//    reference; P = 2^x multiplies the codes of V directly.  P as f16 is cut into hi + mid / 8 + lo / 64
//    of e5m2, three bits each (the upper byte of an f16 IS an e5m2: the cut is a byte permutation, the
//    rest an exact f16 subtraction), relative error <= 2^-9 like a bf16 P.  e5m2 and not e4m3 for its
//    range: a weight keeps its 9 bits down to 2^-21 of the row's reference and vanishes below 2^-30, so
//    a sink token of large weight does not swallow the 10^5 small ones whose weights add up.
//  * the row sum adds P * 2^-ev, unrounded, in fp32 (ev in [-32, 80], see kv8.cuh).
// M is raised lazily (exact maximum of the first tile; later only when some x exceeds 15, so P <= 2^15).
//
// A CTA walks its share of the tiles (kv8.cuh): 4 softmax warps (thread = key of the tile in the
// scores, head dim in the output), one TMA producer warp, one MMA issuer warp.  The producer runs
// ahead across segment ends, so a new segment finds its first tiles in shared memory.  Two CTAs per
// SM (at most 110 KB shared memory, 256 TMEM columns each) hide each other's segment ends.
// Every wait is bounded; on expiry the CTA raises SS_DEV_WAIT_EXPIRED and leaves its tickets in order.
#include <cuda_fp8.h>

#include "kv8.cuh"
#include "tc_ptx.cuh"

namespace ss {
namespace {

using namespace ss::tc;

constexpr float kBias = 7.f, kOver = 15.f;

template <int NR>
struct alignas(16) Ctl8 {
  uint64_t ufull[16], uempty[16];
  uint64_t sfull[2], pready, pfree, qfull;
  uint32_t tmem_base;
  volatile uint32_t abort;
  volatile uint32_t flag[3];
  int last;
  alignas(16) float nm[NR];       // bias - M
  alignas(16) float qf[NR];       // 2^eq * scale * log2(e)
  alignas(16) float smax[4][NR];  // per warp: maxima of a tile; at a segment's end the row sums
};

template <int NR, int D>
struct Cfg8 {
  static constexpr int kUnitBytes = kTok8 * D;             // one K or V tile
  static constexpr int NS = 2 * NR;                        // score columns
  static constexpr int NP = (3 * NR + 15) / 16 * 16;       // weight columns
  static constexpr int kQBytes = NS * D;
  static constexpr int kPBytes = kTok8 * NP;
  static constexpr int kCtlBytes = (sizeof(Ctl8<NR>) + 127) / 128 * 128;
  static constexpr int kRest = (kQBytes + 1023) / 1024 * 1024 + kPBytes + kCtlBytes;
  // head dim 64: the output MMA's upper 64 rows read one unit further on (results never used), the
  // last unit's inside this window too
  static constexpr int kAfter = kRest > kUnitBytes ? kRest : kUnitBytes;
  static constexpr int kUnits0 = (112 * 1024 - kAfter) / kUnitBytes;
  static constexpr int kUnits = kUnits0 > 12 ? 12 : kUnits0;
  static constexpr int kOffQ = kUnits * kUnitBytes;
  static constexpr int kOffP = kOffQ + (kQBytes + 1023) / 1024 * 1024;
  static constexpr int kOffCtl = kOffP + kPBytes;
  static constexpr int kSmem = kOffQ + kAfter;
  static constexpr int kCols = 2 * NS + NP;
  static constexpr uint32_t kTmemCols = kCols <= 64 ? 64 : kCols <= 128 ? 128 : 256;
  static constexpr uint32_t kColO = 2 * NS;
  static_assert(kUnits >= 4 && kCols <= 256, "shape");
};

constexpr int kThreads8 = 192;

__device__ __forceinline__ void mma8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// kind::f8f6f4 -> fp32: format 0 = e4m3, 1 = e5m2
__host__ __device__ constexpr uint32_t idesc8(int N, int b_format, bool mn_major) {
  return (1u << 4) | ((uint32_t)b_format << 10) | ((mn_major ? 3u : 0u) << 15) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(128 >> 4) << 24);
}
// Shared-memory descriptors of tiles with rows of D bytes, swizzled over 128 or 64 bytes; 8-row atoms
// 8 * D bytes apart.  As MN-major operand the row is the MN axis (lbo: the next D elements).
template <int D>
__device__ __forceinline__ uint64_t desc8(uint32_t saddr, uint32_t lbo) {
  return (uint64_t)((saddr >> 4) & 0x3FFF) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)((8 * D) >> 4) << 32) |
         (1ull << 46) | ((D == 128 ? 2ull : 4ull) << 61);
}
__device__ __forceinline__ float2 mul2_f(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(d)
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return reinterpret_cast<float2&>(d);
}
__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }

// Two values of a weight pair's residue: (w - cut) * 8 with cut = w's upper bytes, exact in f16.
__device__ __forceinline__ uint32_t residue(uint32_t w) {
  return h2_bits(__hmul2(__hsub2(bits_h2(w), bits_h2(w & 0xff00ff00u)), __float2half2_rn(8.f)));
}

template <int NR, int D>
__global__ void __launch_bounds__(kThreads8, 2)
attn8_tc_kernel(const __grid_constant__ Attn8Params p, const __grid_constant__ CUtensorMap tmK,
                const __grid_constant__ CUtensorMap tmV) {
  using C = Cfg8<NR, D>;
  constexpr int UNITS = C::kUnits, NS = C::NS, NP = C::NP;
  extern __shared__ __align__(1024) uint8_t smem[];
  Ctl8<NR>* ctl = reinterpret_cast<Ctl8<NR>*>(smem + C::kOffCtl);
  uint8_t* q_s = smem + C::kOffQ;
  uint8_t* p_s = smem + C::kOffP;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kProducerWarp = 4, kMmaWarp = 5;

  if (warp == kProducerWarp) {
    if (lane == 0) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&tmK) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&tmV) : "memory");
      for (int u = 0; u < UNITS; ++u) {
        mbar_init(&ctl->ufull[u], 1);
        mbar_init(&ctl->uempty[u], 1);
      }
      mbar_init(&ctl->sfull[0], 1);
      mbar_init(&ctl->sfull[1], 1);
      mbar_init(&ctl->pready, 128);
      mbar_init(&ctl->pfree, 1);
      mbar_init(&ctl->qfull, 128);
      ctl->abort = 0;
      ctl->flag[0] = ctl->flag[1] = ctl->flag[2] = 0;
      fence_barrier_init();
    }
  }
  // (tensor memory is taken after the wait: the kernel in front may still be about to allocate its own)
  pdl_wait_prior();
  pdl_launch_dependents();
  if (warp == kProducerWarp) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(C::kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const Share8 share = find_share8(p);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;
  auto mwait = [&](uint64_t* bar, uint32_t parity) {
    return mbar_wait_abortable(bar, parity, &ctl->abort, p.status);
  };
  long long base;
  Seg8 g;
  bool more = seg_first8(p, share, &base, &g);

  if (warp == kProducerWarp) {
    // ===== TMA producer =====
    // Pages of a tile or more, and dense caches: one box per tile, by lane 0.  Smaller pages (8 to 64
    // tokens): lane i copies page i of the tile; a page is a whole number of swizzle atoms, so the boxes
    // side by side have the layout of one.  The swizzle atom (8 rows) is also why other page sizes
    // take the CUDA-core kernel.  Pages past the request's last token are not looked up.
    const uint64_t pol = p.row_tiles > 1 ? l2_evict_normal_policy() : l2_evict_first_policy();
    const bool small = p.kv.page_table && p.kv.page_size < kTok8;
    const int ps = small ? p.kv.page_size : kTok8;
    const bool mine = lane < kTok8 / ps;
    int j = 0;
    bool ok = true;
    for (; more && ok; more = seg_next8(p, share, &base, &g)) {
      int inner = 0, outer = 0;
      auto look = [&](int t) {  // this lane's page of tile t
        const int tok = t * kTok8 + lane * ps;
        outer = p.kv.n_outer;   // outside the tensor: reads as zeros
        inner = 0;
        if (!mine || t >= g.t1 || tok >= g.len) return;
        const int id = outer8(p.kv, g.b, tok, &inner);
        if (id >= 0) outer = id;
        else atomicOr(p.status, SS_DEV_BAD_PAGE);
      };
      look(g.t0);
      for (int t = g.t0; t < g.t1 && ok; ++t) {
        for (int kv = 0; kv < 2; ++kv, ++j) {
          const int u = j % UNITS;
          int go = 1;
          if (lane == 0) {
            go = mwait(&ctl->uempty[u], ((j / UNITS) & 1) ^ 1);
            if (go) mbar_expect_tx(&ctl->ufull[u], C::kUnitBytes);
          }
          ok = __shfl_sync(0xffffffffu, go, 0);  // (also orders the arming before the copies)
          if (!ok) break;
          const uint32_t dst = smem_u32(smem + u * C::kUnitBytes) + lane * ps * D;
          if (mine) tma_load_4d(dst, kv ? &tmV : &tmK, 0, inner, g.kvh, outer, &ctl->ufull[u], pol);
        }
        look(t + 1);
      }
    }
    if (lane == 0 && ctl->abort) {  // let the copies in flight land before the CTA leaves (bounded)
      const unsigned long long t0 = gtime_ns();
      for (int i = max(0, j - UNITS); i < j; ++i)
        while (!mbar_try_wait(&ctl->ufull[i % UNITS], (i / UNITS) & 1) && gtime_ns() - t0 < kWaitNs) {
        }
    }
  } else if (warp == kMmaWarp) {
    // ===== MMA issuer: polls for whichever of its two next operations can go =====
    constexpr uint32_t idesc_qk = idesc8(NS, 0, false), idesc_pv = idesc8(NP, 1, true);
    const bool leader = elect_one();
    const uint32_t ring = smem_u32(smem), q_addr = smem_u32(q_s), p_addr = smem_u32(p_s);
    int it0 = 0, seg = 0;  // tiles and segments before this one
    bool ok = true;
    for (; more && ok; more = seg_next8(p, share, &base, &g), ++seg) {
      const int n = g.t1 - g.t0;
      int qi = 0, pi = 0;
      bool q_there = false;
      unsigned long long t0 = gtime_ns();
      uint32_t spins = 0;
      while (pi < n) {
        bool did = false;
        if (qi < n && qi < pi + 2) {
          const int it = it0 + qi, jk = 2 * it;
          if (!q_there) q_there = __all_sync(0xffffffffu, mbar_test(&ctl->qfull, seg & 1));
          if (q_there && __all_sync(0xffffffffu, mbar_test(&ctl->ufull[jk % UNITS], (jk / UNITS) & 1))) {
            tc_fence_after();
            const uint32_t k_addr = ring + (jk % UNITS) * C::kUnitBytes;
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < D / 32; ++kk)
                mma8(tmem + (it & 1) * NS, desc8<D>(k_addr + kk * 32, 16), desc8<D>(q_addr + kk * 32, 16), idesc_qk, kk > 0);
              tc_commit(&ctl->uempty[jk % UNITS]);
              tc_commit(&ctl->sfull[it & 1]);
            }
            __syncwarp();
            ++qi;
            did = true;
          }
        }
        if (pi < qi) {
          const int it = it0 + pi, jv = 2 * it + 1;
          if (__all_sync(0xffffffffu, mbar_test(&ctl->pready, it & 1) &&
                                          mbar_test(&ctl->ufull[jv % UNITS], (jv / UNITS) & 1))) {
            tc_fence_after();
            const uint32_t v_addr = ring + (jv % UNITS) * C::kUnitBytes;
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < kTok8 / 32; ++kk)
                mma8(tmem + C::kColO, desc8<D>(v_addr + kk * 32 * D, C::kUnitBytes),
                     desc_mnmajor_plain(p_addr + kk * 512, 128, kTok8 * 16), idesc_pv, pi > 0 || kk > 0);
              tc_commit(&ctl->uempty[jv % UNITS]);
              tc_commit(&ctl->pfree);
            }
            __syncwarp();
            ++pi;
            did = true;
          }
        }
        if (did) {
          spins = 0;
          t0 = gtime_ns();
        } else if ((++spins & 255u) == 0) {
          const bool stop = ctl->abort != 0 || gtime_ns() - t0 > kWaitNs;
          if (__any_sync(0xffffffffu, stop)) {
            if (lane == 0 && ctl->abort == 0) {
              ctl->abort = 1;
              atomicOr(p.status, SS_DEV_WAIT_EXPIRED);
            }
            ok = false;
            break;
          }
        }
      }
      it0 += n;
    }
  } else {
    // ===== softmax warps =====
    // A wait that gives up makes the warp `dead`: it keeps walking the segments, barriers and tickets,
    // so nobody is left waiting, and touches nothing else.
    const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
    bool dead = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead && !mwait(bar, parity)) dead = true;
      dead = __any_sync(0xffffffffu, dead);
    };
    put_empty8(p, tid, 128);

    // Q: 128 / NR threads per row, kE values each
    constexpr int TPR = 128 / NR, kE = D / TPR, kQL = kE / 4;
    const int q_row = tid / TPR, q_part = tid % TPR;
    uint2 q_raw[kQL];
    auto q_load = [&](const Seg8& s) {
      const int rg = s.row0 + q_row, h = s.kvh * p.G + rg / p.T_q, t = rg % p.T_q;
      const __nv_bfloat16* src = p.Q + s.b * p.q_sb + h * p.q_sh + t * p.q_st + q_part * kE;
#pragma unroll
      for (int i = 0; i < kQL; ++i)
        q_raw[i] = q_row < s.nrows ? *reinterpret_cast<const uint2*>(src + i * 4) : make_uint2(0, 0);
    };
    auto q_store = [&]() {
      uint32_t w[2 * kQL], top = 0;
#pragma unroll
      for (int i = 0; i < kQL; ++i) {
        w[2 * i] = q_raw[i].x;
        w[2 * i + 1] = q_raw[i].y;
      }
#pragma unroll
      for (int i = 0; i < 2 * kQL; ++i) {
        const uint32_t a = w[i] & 0x7fffu, b = (w[i] >> 16) & 0x7fffu;
        if (a < 0x7f80u) top = max(top, a);
        if (b < 0x7f80u) top = max(top, b);
      }
#pragma unroll
      for (int o = TPR / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int eq = max(-100, min(119, (int)(top >> 7) - 127 - 7));  // |q| * 2^-eq < 256
      const float inv = pow2_8(-eq);
      uint32_t hi[kE / 4], lo[kE / 4];
#pragma unroll
      for (int i = 0; i < kE / 4; ++i) {
        uint32_t h4 = 0, l4 = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t two = w[2 * i + k];
          // (an infinite or NaN query makes its scores NaN)
          float2 v = make_float2(__uint_as_float(two << 16) * inv, __uint_as_float(two & 0xffff0000u) * inv);
          if ((two & 0x7f80u) == 0x7f80u) v.x = __int_as_float(0x7fffffff);
          if ((two & 0x7f800000u) == 0x7f800000u) v.y = __int_as_float(0x7fffffff);
          const uint32_t c = __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
          const __half2_raw hr = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
          const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hr));
          const uint32_t r = __nv_cvt_float2_to_fp8x2(make_float2((v.x - back.x) * 16.f, (v.y - back.y) * 16.f),
                                                      __NV_SATFINITE, __NV_E4M3);
          h4 |= c << (16 * k);
          l4 |= r << (16 * k);
        }
        hi[i] = h4;
        lo[i] = l4;
      }
      // operand row n, 16-byte piece c at n * D + ((c ^ swizzle(n)) * 16); rows r and r + 8 of a group of
      // 16 hold hi and lo of the same query row
      const int n = 16 * (q_row / 8) + q_row % 8;
#pragma unroll
      for (int term = 0; term < 2; ++term) {
        const int nn = n + 8 * term;
        const int sw = D == 128 ? (nn & 7) : ((nn >> 1) & 3);
#pragma unroll
        for (int i = 0; i < kE / 4; ++i) {
          const int byte = q_part * kE + i * 4;
          *reinterpret_cast<uint32_t*>(q_s + nn * D + (((byte >> 4) ^ sw) << 4) + (byte & 15)) = term ? lo[i] : hi[i];
        }
      }
      if (q_part == 0) ctl->qf[q_row] = pow2_8(eq) * p.scale_log2;
      fence_proxy_async();
      mbar_arrive(&ctl->qfull);
    };

    // Scale bytes of this thread's key, fetched a tile ahead (and its page id two tiles ahead).
    struct Ahead {
      int outer, inner;      // where the key of the tile after next lives
      uint32_t ek, ev;       // bytes of the next tile's key
    } ah;
    auto ah_look = [&](const Seg8& s, int t) {
      const int tok = t * kTok8 + tid;
      ah.outer = -1;
      ah.inner = 0;
      if (t < s.t1 && tok < s.len) ah.outer = outer8(p.kv, s.b, tok, &ah.inner);
    };
    auto ah_fetch = [&](const Seg8& s) {
      ah.ek = ah.ev = 127;   // (a key that is not there, or in a page outside the pool: value 0)
      if (ah.outer >= 0) {
        ah.ek = p.kv.Ks[ah.outer * p.kv.ks_sb + s.kvh * p.kv.ks_sh + ah.inner * p.kv.ks_st];
        ah.ev = p.kv.Vs[ah.outer * p.kv.vs_sb + s.kvh * p.kv.vs_sh + ah.inner * p.kv.vs_st];
      }
    };
    if (more) {
      ah_look(g, g.t0);
      q_load(g);
      ah_fetch(g);
      ah_look(g, g.t0 + 1);
    }

    int it = 0;
    while (more) {
      q_store();
      float2 lsum[NR / 2];
#pragma unroll
      for (int r = 0; r < NR / 2; ++r) lsum[r] = make_float2(0.f, 0.f);
      for (int t = g.t0; t < g.t1; ++t, ++it) {
        const float kf = scale8(ah.ek), evf = (float)(int)ah.ev - 127.f, vinv = scale8(254u - ah.ev);
        ah_fetch(g);
        ah_look(g, t + 2);
        const int n_valid = min(kTok8, g.len - t * kTok8);
        const bool key_ok = tid < n_valid;
        wait(&ctl->sfull[it & 1], (it >> 1) & 1);
        tc_fence_after();
        if (n_valid < kTok8) {
          // tokens past the length may hold anything; their weights are 0, so V must be finite there
          const int jv = 2 * it + 1;
          wait(&ctl->ufull[jv % UNITS], (jv / UNITS) & 1);
          if (!dead) {
            uint4* v = reinterpret_cast<uint4*>(smem + (jv % UNITS) * C::kUnitBytes);
            for (int i = n_valid * (D / 16) + tid; i < kTok8 * (D / 16); i += 128) v[i] = make_uint4(0, 0, 0, 0);
          }
        }
        // x[r] = s2 + ev (first tile) or s2 + ev - M + bias
        float x[NR];
        const bool first = t == g.t0;
        if (!dead) {
#pragma unroll
          for (int q = 0; q < NR / 8; ++q) {
            uint32_t raw[16];
            tmem_ld16(tmem + lane_off + (it & 1) * NS + q * 16, raw);
            tc_wait_ld();
#pragma unroll
            for (int c = 0; c < 8; c += 4) {
              const float4 qf = *reinterpret_cast<const float4*>(&ctl->qf[q * 8 + c]);
              float4 nm = make_float4(0.f, 0.f, 0.f, 0.f);
              if (!first) nm = *reinterpret_cast<const float4*>(&ctl->nm[q * 8 + c]);
              const float qs[4] = {qf.x, qf.y, qf.z, qf.w}, ns[4] = {nm.x, nm.y, nm.z, nm.w};
#pragma unroll
              for (int k = 0; k < 4; k += 2) {
                const float2 hi = make_float2(__uint_as_float(raw[c + k]), __uint_as_float(raw[c + k + 1]));
                const float2 lo = make_float2(__uint_as_float(raw[8 + c + k]), __uint_as_float(raw[8 + c + k + 1]));
                const float2 s = mul2_f(fma2_f(lo, make_float2(0.0625f, 0.0625f), hi), make_float2(qs[k], qs[k + 1]));
                const float2 y = fma2_f(s, make_float2(kf, kf), add2_f(make_float2(ns[k], ns[k + 1]), make_float2(evf, evf)));
                x[q * 8 + c + k] = y.x;
                x[q * 8 + c + k + 1] = y.y;
              }
            }
          }
        }
        auto tile_max = [&]() {  // exact maxima of x over the tile's keys, all four warps
          if (!dead) {
            float mine = -INFINITY;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              const float m = redux_max(key_ok ? x[r] : -INFINITY);
              if (lane == r) mine = m;
            }
            if (lane < NR) ctl->smax[warp][lane] = mine;
          }
          bar8(128);
        };
        auto top4 = [&](int r) {
          return fmaxf(fmaxf(ctl->smax[0][r], ctl->smax[1][r]), fmaxf(ctl->smax[2][r], ctl->smax[3][r]));
        };
        if (first) {
          tile_max();
          if (!dead) {
#pragma unroll
            for (int r = 0; r < NR; ++r) x[r] += kBias - top4(r);
            if (tid < NR) ctl->nm[tid] = kBias - top4(tid);  // (read from the next tile on)
          }
          if (tid == 0) ctl->flag[(it + 1) % 3] = 0;
          bar8(128);
        } else {
          float mx = -INFINITY;
          if (!dead) {
#pragma unroll
            for (int r = 0; r < NR; r += 2) mx = max3_f(mx, x[r], x[r + 1]);
          }
          if (tid == 0) ctl->flag[(it + 1) % 3] = 0;
          if (__any_sync(0xffffffffu, key_ok && mx > kOver) && lane == 0) ctl->flag[it % 3] = 1;
          bar8(128);
          if (ctl->flag[it % 3]) {
            // ---- raise the references to the exact maxima: rescale O^T and the row sums (rare) ----
            tile_max();
            wait(&ctl->pfree, (it - 1) & 1);  // the output MMAs of the tile before have retired
            tc_fence_after();
            if (!dead) {
#pragma unroll
              for (int r = 0; r < NR; ++r) {
                const float up = fmaxf(0.f, top4(r) - kBias);  // M rises by this much
                x[r] -= up;
                if (r & 1) lsum[r / 2].y *= ex2_ftz(-up);
                else lsum[r / 2].x *= ex2_ftz(-up);
              }
#pragma unroll
              for (int q = 0; q < NP / 16; ++q) {
                uint32_t o[16];
                tmem_ld16(tmem + lane_off + C::kColO + q * 16, o);
                tc_wait_ld();
#pragma unroll
                for (int c = 0; c < 16; ++c)
                  o[c] = __float_as_uint(__uint_as_float(o[c]) * ex2_ftz(-fmaxf(0.f, top4((q * 16 + c) % NR) - kBias)));
                tmem_st16(tmem + lane_off + C::kColO + q * 16, o);
              }
              tc_wait_st();
            }
            bar8(128);
            if (tid < NR && !dead) ctl->nm[tid] -= fmaxf(0.f, top4(tid) - kBias);
            bar8(128);
          }
        }
        if (it > 0 && !first) wait(&ctl->pfree, (it - 1) & 1);  // P^T has been consumed
        if (!dead) {
          uint32_t w[NR / 2];
#pragma unroll
          for (int r = 0; r < NR; r += 2) {
            float2 e = make_float2(ex2_ftz(x[r]), ex2_ftz(x[r + 1]));
            if (n_valid < kTok8) e = key_ok ? e : make_float2(0.f, 0.f);
            lsum[r / 2] = fma2_f(e, make_float2(vinv, vinv), lsum[r / 2]);
            w[r / 2] = h2_bits(__float22half2_rn(e));
          }
          // columns term * NR + r, 16 to a 16-byte piece per key
          uint32_t piece[NP / 4];
#pragma unroll
          for (int c = 0; c < NP / 4; ++c) piece[c] = 0;
#pragma unroll
          for (int r = 0; r < NR; r += 4) {
            const uint32_t a = w[r / 2], b = w[r / 2 + 1];
            const uint32_t a1 = residue(a), b1 = residue(b);
            const uint32_t a2 = residue(a1) + 0x00800080u, b2 = residue(b1) + 0x00800080u;  // (the last term rounds)
            piece[r / 4] = __byte_perm(a, b, 0x7531);
            piece[(NR + r) / 4] = __byte_perm(a1, b1, 0x7531);
            piece[(2 * NR + r) / 4] = __byte_perm(a2, b2, 0x7531);
          }
#pragma unroll
          for (int q = 0; q < NP / 16; ++q)
            *reinterpret_cast<uint4*>(p_s + q * (kTok8 * 16) + tid * 16) =
                make_uint4(piece[4 * q], piece[4 * q + 1], piece[4 * q + 2], piece[4 * q + 3]);
          fence_proxy_async();
          tc_fence_before();
        }
        mbar_arrive(&ctl->pready);
      }

      // ---- the segment's end: what the next one needs is fetched first ----
      const Seg8 done = g;
      more = seg_next8(p, share, &base, &g);
      if (more) {
        ah_look(g, g.t0);
        q_load(g);
        ah_fetch(g);
        ah_look(g, g.t0 + 1);
      }
      // row sums: halve the rows a lane holds at every step, lane / (32 / NR) is the row in the end
      {
        float v[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) v[r] = (r & 1) ? lsum[r / 2].y : lsum[r / 2].x;
        int n = NR;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
          if (n > 1) {
            n /= 2;
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < NR / 2; ++i) {
              if (i < n) {
                const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
              }
            }
          } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
          }
        }
        bar8(128);  // (every thread is done with smax as maxima)
        if (lane % (32 / NR) == 0) ctl->smax[warp][lane / (32 / NR)] = v[0];
      }
      wait(&ctl->pfree, (it - 1) & 1);
      tc_fence_after();
      bar8(128);
      const bool whole = done.t0 == 0 && done.t1 == done.n;
      float* slot = slot8(p, share, done.start, blockIdx.x);
      const float (*sums)[NR] = ctl->smax;
      auto row_l = [&](int r) { return (sums[0][r] + sums[1][r]) + (sums[2][r] + sums[3][r]); };
      if (!dead) {
        if (tid < done.nrows) {
          const float m = -ctl->nm[tid], l = row_l(tid);  // the sums are of 2^(s2 - M + bias)
          if (whole) put_ml8(p, done, tid, m, l);
          else reinterpret_cast<float2*>(slot)[tid] = make_float2(m, l);
        }
#pragma unroll
        for (int q = 0; q < NR / 8; ++q) {
          uint32_t o[3][8];
#pragma unroll
          for (int k = 0; k < 3; ++k)
            asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(o[k][0]), "=r"(o[k][1]), "=r"(o[k][2]), "=r"(o[k][3]), "=r"(o[k][4]), "=r"(o[k][5]),
                           "=r"(o[k][6]), "=r"(o[k][7])
                         : "r"(tmem + lane_off + C::kColO + k * NR + q * 8)
                         : "memory");
          tc_wait_ld();
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const int r = q * 8 + c;
            if (r < done.nrows && tid < D) {
              const float a = fmaf(__uint_as_float(o[2][c]), 1.f / 64.f,
                                   fmaf(__uint_as_float(o[1][c]), 0.125f, __uint_as_float(o[0][c])));
              if (whole) put_a8(p, done, r, tid, row_l(r), a);
              else slot[2 * p.rows_per_tile + r * D + tid] = a;
            }
          }
        }
      }
      tc_fence_before();
      if (!whole) join8<D>(p, share, done, tid, &ctl->last);
      bar8(128);  // sums, references and Q may be written anew
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kProducerWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
}

template <int NR, int D>
cudaError_t prepare8() {
  return cudaFuncSetAttribute(attn8_tc_kernel<NR, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg8<NR, D>::kSmem);
}
template <int NR, int D>
cudaError_t launch8(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  return launch_kernel(attn8_tc_kernel<NR, D>, dim3(kCtas8), dim3(kThreads8), Cfg8<NR, D>::kSmem, s, pdl, p, tmK, tmV);
}

}  // namespace

cudaError_t attn8_tc_prepare() {
  cudaError_t e = prepare8<8, 128>();
  if (e == cudaSuccess) e = prepare8<16, 128>();
  if (e == cudaSuccess) e = prepare8<32, 128>();
  if (e == cudaSuccess) e = prepare8<8, 64>();
  if (e == cudaSuccess) e = prepare8<16, 64>();
  if (e == cudaSuccess) e = prepare8<32, 64>();
  return e;
}

cudaError_t launch_attn8_tc(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  const int rows = p.rows_per_tile;
  if (p.d == 128)
    return rows <= 8 ? launch8<8, 128>(p, tmK, tmV, s, pdl)
                     : rows <= 16 ? launch8<16, 128>(p, tmK, tmV, s, pdl) : launch8<32, 128>(p, tmK, tmV, s, pdl);
  return rows <= 8 ? launch8<8, 64>(p, tmK, tmV, s, pdl)
                   : rows <= 16 ? launch8<16, 64>(p, tmK, tmV, s, pdl) : launch8<32, 64>(p, tmK, tmV, s, pdl);
}

}  // namespace ss
