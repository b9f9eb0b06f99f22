// Attention over the 8-bit KV cache on the tensor cores: the codes go from HBM to the MMA as they
// are, nothing dequantises them.
//
//   S^T = K Q^T    M = 128 keys of the tile, N = rows, K = d         (d / 32 steps, e4m3 x e4m3)
//   O^T = V^T P^T  M = 128 head dims,        N = rows, K = 128 keys  (4 steps, e4m3 x e5m2)
//
// as in the bf16 kernel with the keys on M; tcgen05.mma kind::f8f6f4 takes both operands in 8 bits, so
// Q and P are split into terms of 8 bits whose products add up in the accumulators (tensor work is not
// what bounds this kernel):
//  * Q row * 2^-eq (maximum in (224, 448]) = hi + lo, both e4m3.  bf16 has 8 significant bits and a term
//    holds 4, so the split is exact as long as lo's last bit is on e4m3's smallest step, 2^-9: for values from 1/4
//    on, 2^-9.8 of the row's maximum; below it is off by at most 2^-10, 2^-17.8 of the maximum.
//    The score is S * 2^eq * 2^ek * scale: all factors powers of two but the caller's, the sums in fp32.
//  * weights.  x = s2 + ev - M + 7 with s2 the score in base 2, ev the key's value exponent, M the row's
//    reference; P = 2^x multiplies the codes of V directly.  P as f16 is cut into hi + mid / 8 + lo / 64 of
//    e5m2, three bits each (the upper byte of an f16 IS an e5m2: the cut is a byte permutation, the rest
//    an exact f16 subtraction), relative error <= 1.1 * 2^-9, f16's own rounding in it.  e5m2 and not e4m3 for its range: a weight keeps
//    its 9 bits down to 2^-20 of the row's reference and is off by at most 1.25 * 2^-30 of it below, so a sink
//    token of large weight does not swallow the 10^5 small ones whose weights add up.
//  * the row sum adds P * 2^-ev, unrounded, in fp32 (ev in [-32, 80], see kv8.cuh).
// The terms of P stand side by side on the N axis (one pass of the MMA over V), and so do those of Q: as
// further steps along K they spared additions, but K's tile was read from shared memory twice (40 rows,
// 16 x 16384 tokens: 155 us against 149; 32 rows, 16 x 32768: 182.5 against 181).
// M is raised lazily (exact maximum of the first tile; later only when some x exceeds 15, so P <= 2^15:
// eight binades of room, since one raise stops all rows of the CTA; with two binades - and unscaled
// terms, one instruction less per weight - every second tile of a 32-row round raised, 281 -> 438 us).
//
// A CTA walks its share of the tiles (kv8.cuh): 4 softmax warps (thread = key of the tile in the
// scores, head dim in the output; with a second set of four for 32 rows 64 rows took 185 us against 179),
// one TMA producer warp, one MMA issuer warp.  The producer runs ahead across segment ends, so a new
// segment finds its first tiles in shared memory.  Two or three CTAs per SM hide each other's segment ends.
// Every wait is bounded; on expiry the CTA raises SS_DEV_WAIT_EXPIRED and returns.
#include <cuda_fp8.h>

#include <type_traits>

#include "kv8_tc.cuh"

namespace ss {
namespace {

using namespace ss::tc;

constexpr float kBias = 7.f, kOver = 15.f;

template <int NQ>
struct alignas(16) Ctl8 {
  uint64_t ufull[16], uempty[16];
  uint64_t sfull[2], pready, pfree, qfull;
  uint32_t tmem_base;
  volatile uint32_t abort;
  int has[2];                     // the softmax warps' current and next segment (in use by turns)
  Seg8 seg[2];
  Share8 share;
  alignas(16) float nm[NQ];       // bias - M
  alignas(16) float qf[NQ];       // 2^eq * scale * log2(e)
  alignas(16) float up[NQ];       // rise of the references; at a segment's end 1 / row sum
  alignas(16) float smax[4][NQ];  // per warp: maxima of a tile; at a segment's end the row sums
};

// What attention over a window (span8 in kv8.cuh) keeps besides.
template <int NQ>
struct CtlWin8 : Ctl8<NQ> {
  int unset;                      // rows without a reference
  alignas(16) int pos[NQ];        // the rows' positions
};

// NR = rows, D = head dim, WIN = over a window.
template <int NR, int D, bool WIN>
struct Cfg8 {
  static constexpr int kSoft = 128, kThreads = kSoft + 64; // softmax threads, all threads
  static constexpr int NQ = NR == 24 ? 32 : NR;            // rows of the Q operand (N has to be a multiple of 16)
  static constexpr int kUnitBytes = kTok8 * D;             // one K or V tile
  static constexpr int NS = 2 * NQ;                    // score columns, hi and lo
  static constexpr int NP = (3 * NR + 15) / 16 * 16;       // weight columns
  static constexpr int kQBytes = 2 * NQ * D;
  static constexpr int kPBytes = kTok8 * NP;
  using Ctl = std::conditional_t<WIN, CtlWin8<NQ>, Ctl8<NQ>>;
  static constexpr int kCtlBytes = (sizeof(Ctl) + 127) / 128 * 128;
  static constexpr int kPartsBytes = WIN ? Parts8<NQ, D, NR == 8>::kBytes : 0;   // (clusters)
  static constexpr int kRest = (kQBytes + 1023) / 1024 * 1024 + kPBytes + kCtlBytes + kPartsBytes;
  // head dim 64: the output MMA's upper 64 rows read one unit further on (results never used), the
  // last unit's inside this window too
  static constexpr int kAfter = D == 64 && kRest < kUnitBytes ? kUnitBytes : kRest;
  // Resident CTAs.  Head dim 64 has half the bytes per tile for the same chain of steps, so a third CTA
  // pays (16 x 32768 tokens in pages of 16, 4 rows: 134 -> 107 us; 16 rows, pages of 64: 112 -> 97); at
  // head dim 128 its shorter rings cost more than it gives (166 -> 170 us).
  static constexpr int kPerSM = D == 64 && NR <= kFew8 ? 3 : 2;
  static constexpr int kUnits0 = ((kPerSM == 3 ? 74 : 112) * 1024 - kAfter) / kUnitBytes;
  static constexpr int kUnits = kUnits0 > 12 ? 12 : kUnits0;
  static constexpr int kOffQ = kUnits * kUnitBytes;
  static constexpr int kOffP = kOffQ + (kQBytes + 1023) / 1024 * 1024;
  static constexpr int kOffCtl = kOffP + kPBytes;
  static constexpr int kOffParts = kOffCtl + kCtlBytes;
  static constexpr int kSmem = kOffQ + kAfter;
  static constexpr int kCols = 2 * NS + NP;
  static constexpr uint32_t kTmemCols = kCols <= 64 ? 64 : kCols <= 128 ? 128 : 256;
  static constexpr uint32_t kColO = 2 * NS;
  static_assert(kUnits >= 4 && kCols <= 256 && NR % 8 == 0 && kUnits * kUnitBytes >= NQ * (D + 5) * 4, "shape");
};

// A descriptor's low word holds the address / 16 (and the LBO above it), so the operands of the steps of
// a tile differ by an addition there; the high word is the same for all.
__device__ __forceinline__ void mma8(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                     uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %5, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
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
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }

// What a pair of weights leaves when its upper bytes are cut off, times 8, exact in f16.
__device__ __forceinline__ uint32_t residue(uint32_t w) {
  return h2_bits(__hmul2(__hsub2(bits_h2(w), bits_h2(w & 0xff00ff00u)), __float2half2_rn(8.f)));
}
// WIN: over a window; CL: a unit is one cluster's (kCluster8), each CTA has one segment.
template <int NR, int D, bool WIN, bool CL>
__global__ void __launch_bounds__(Cfg8<NR, D, WIN>::kThreads, Cfg8<NR, D, WIN>::kPerSM)
attn8_tc_kernel(const __grid_constant__ Attn8Params p, const __grid_constant__ CUtensorMap tmK,
                const __grid_constant__ CUtensorMap tmV) {
  using C = Cfg8<NR, D, WIN>;
  constexpr int UNITS = C::kUnits, NQ = C::NQ, NS = C::NS, NP = C::NP, SOFT = C::kSoft;
  extern __shared__ __align__(1024) uint8_t smem[];
  typename C::Ctl* ctl = reinterpret_cast<typename C::Ctl*>(smem + C::kOffCtl);
  uint8_t* q_s = smem + C::kOffQ;
  uint8_t* p_s = smem + C::kOffP;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kProducerWarp = 4, kMmaWarp = 5;

  // The warp that takes the tensor memory.  Over a window the producer is free of it and of the barrier in front of
  // the roles: its first copies have a chain of dependent loads in front of them that all the rest waits for.
  constexpr int kTmemWarp = WIN ? kMmaWarp : kProducerWarp;

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
      mbar_init(&ctl->pready, SOFT);
      mbar_init(&ctl->pfree, 1);
      mbar_init(&ctl->qfull, SOFT);
      ctl->abort = 0;
      if constexpr (WIN) ctl->unset = 0;
      fence_barrier_init();
    }
    if (WIN) {
      __syncwarp();
      __threadfence_block();
      asm volatile("barrier.cta.arrive 2, %0;" ::"n"(C::kThreads) : "memory");
    }
  }
  Place8 place = {};
  if (CL) place = cluster_place8(p);
  constexpr bool PUSH = CL && NR == 8;
  const Parts8<NQ, D, PUSH> parts(reinterpret_cast<float*>(smem + (PUSH ? C::kOffParts : 0)), p, place);
  auto find = [&]() {
    Share8 s = {};
    if (!CL) s = find_share8<WIN>(p);
    return s;
  };
  auto seg_first = [&](const Share8& s, Seg8* g) { return CL ? cluster_seg8(p, place, g) : seg_first8<WIN>(p, s, g); };
  auto seg_next = [&](const Share8& s, Seg8* g) { return !CL && seg_next8<WIN>(p, s, g); };
  // (tensor memory is taken after the wait: the kernel in front may still be about to allocate its own)
  pdl_wait_prior();
  pdl_launch_dependents();
  if (warp == kTmemWarp) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(C::kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == 0) {
    const Share8 share = find();
    if (lane == 0) {
      ctl->share = share;
      ctl->has[0] = seg_first(share, &ctl->seg[0]);
    }
  }
  if (!WIN) {
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  } else if (warp != kProducerWarp) {
    tc_fence_before();
    asm volatile("barrier.cta.sync 2, %0;" ::"n"(C::kThreads) : "memory");
    tc_fence_after();
  }
  const uint32_t tmem = ctl->tmem_base;
  const Share8& share = ctl->share;
  auto mwait = [&](uint64_t* bar, uint32_t parity) {
    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, &ctl->abort, p.status);
  };

  if (warp == kProducerWarp) {
    // ===== TMA producer =====
    // Pages of a tile or more, and dense caches: one box per tile, by lane 0.  Smaller pages (8 to 64
    // tokens): lane i copies page i of the tile; a page is a whole number of swizzle atoms, so the boxes
    // side by side have the layout of one.  The swizzle atom (8 rows) is also why other page sizes
    // take the CUDA-core kernel.  Pages past the request's last token are not looked up.
    const uint64_t pol = p.row_tiles > 1 ? l2_evict_normal_policy() : l2_evict_first_policy();
    // Over a window lane i copies granule i.
    const bool small = p.kv.page_shift >= 0;
    const int ps = WIN ? 1 << p.gran_log2 : small ? p.kv.page_size : kTok8;
    const bool mine = lane * ps < kTok8;
    int j = 0, u = 0;      // units filled so far, the next one's place in the ring
    uint32_t ph = 1;       // parity of its release
    bool ok = true;
    Seg8 g;
    const Share8 mine_share = WIN ? find() : share;
    for (bool more = seg_first(mine_share, &g); more && ok; more = seg_next(mine_share, &g)) {
      Win8 w = {};
      if (WIN) w = win8(p, g.b);
      int inner = 0, outer = 0;
      auto look = [&](int t) {  // this lane's page of tile t
        const int tok = t * kTok8 + lane * ps;
        outer = p.kv.n_outer;   // outside the tensor: reads as zeros
        inner = 0;
        if (!mine || t >= g.t1 || tok >= g.len) return;
        int id = g.b;
        if (WIN) {
          inner = win_token8(w, tok);
          if (p.kv.page_table) id = page8(p.kv, g.b, &inner);
        } else if (!p.kv.page_table) {
          inner = tok;
        } else {
          const int pg = small ? tok >> p.kv.page_shift : p.kv.page_tiles == 1 ? t : t / p.kv.page_tiles;
          if (!small) inner = tok - pg * p.kv.page_size;
          id = p.kv.page_table[(int64_t)g.b * p.kv.pages_per_req + pg];
        }
        if (id >= 0 && id < p.kv.n_outer) outer = id;
        else atomicOr(p.status, SS_DEV_BAD_PAGE);
      };
      look(g.t0);
      for (int t = g.t0; t < g.t1 && ok; ++t) {
        for (int kv = 0; kv < 2; ++kv, ++j) {
          int go = 1;
          if (lane == 0) {
            go = mwait(&ctl->uempty[u], ph);
            if (go) mbar_expect_tx(&ctl->ufull[u], C::kUnitBytes);
          }
          ok = __shfl_sync(0xffffffffu, go, 0);  // (also orders the arming before the copies)
          if (!ok) break;
          const uint32_t dst = smem_u32(smem + u * C::kUnitBytes) + lane * ps * D;
          if (mine) {
            if (kv) tma_load_4d(dst, &tmV, 0, inner, g.kvh, outer, &ctl->ufull[u], pol);
            else tma_load_4d(dst, &tmK, 0, inner, g.kvh, outer, &ctl->ufull[u], pol);
          }
          if (++u == UNITS) {
            u = 0;
            ph ^= 1;
          }
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
    if constexpr (WIN) {
      __syncwarp();
      if (p.depth) check_depths8(p);
    }
  } else if (warp == kMmaWarp) {
    // ===== MMA issuer: polls for whichever of its two next operations can go =====
    constexpr uint32_t idesc_qk = idesc8(NS, 0, false), idesc_pv = idesc8(NP, 1, true);
    const bool leader = elect_one();
    const uint64_t k_desc = desc8<D>(smem_u32(smem), 16), v_desc = desc8<D>(smem_u32(smem), C::kUnitBytes),
                   q_desc = desc8<D>(smem_u32(q_s), 16), p_desc = desc_mnmajor_plain(smem_u32(p_s), 128, kTok8 * 16);
    const uint32_t k_lo = (uint32_t)k_desc, v_lo = (uint32_t)v_desc, q_lo = (uint32_t)q_desc, p_lo = (uint32_t)p_desc;
    const uint32_t k_hi = (uint32_t)(k_desc >> 32), v_hi = (uint32_t)(v_desc >> 32), q_hi = (uint32_t)(q_desc >> 32),
                   p_hi = (uint32_t)(p_desc >> 32);
    // ring positions of the next score MMAs' K and of the next output MMAs' V, with their phases
    int uk = 0, uv = 1;
    uint32_t phk = 0, phv = 0;
    auto step = [&](int& u, uint32_t& ph) {
      u += 2;
      if (u >= UNITS) {
        u -= UNITS;
        ph ^= 1;
      }
    };
    int it0 = 0, seg = 0;  // tiles and segments before this one
    bool ok = true;
    Seg8 g = ctl->seg[0];
    for (bool more = ctl->has[0]; more && ok; more = seg_next(share, &g), ++seg) {
      const int n = g.t1 - g.t0;
      int qi = 0, pi = 0;
      bool q_there = false;
      unsigned long long t0 = gtime_ns();
      uint32_t spins = 0;
      while (pi < n) {
        bool did = false;
        if (qi < n && qi < pi + 2) {
          const int it = it0 + qi;
          if (!q_there) q_there = __all_sync(0xffffffffu, mbar_test(&ctl->qfull, seg & 1));
          if (q_there && __all_sync(0xffffffffu, mbar_test(&ctl->ufull[uk], phk))) {
            tc_fence_after();
            if (leader) {
              const uint32_t a = k_lo + uk * (C::kUnitBytes / 16), d_s = tmem + (it & 1) * NS;
#pragma unroll
              for (int kk = 0; kk < D / 32; ++kk)
                mma8(d_s, a + kk * 2, k_hi, q_lo + kk * 2, q_hi, idesc_qk, kk > 0);
              tc_commit(&ctl->uempty[uk]);
              tc_commit(&ctl->sfull[it & 1]);
            }
            __syncwarp();
            step(uk, phk);
            ++qi;
            did = true;
          }
        }
        if (pi < qi) {
          const int it = it0 + pi;
          // with the scores two tiles ahead nothing but this can go: sleep on it instead of polling
          bool go = true;
          if (qi == n || qi == pi + 2) {
            ok = mwait(&ctl->pready, it & 1) && mwait(&ctl->ufull[uv], phv);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
          } else {
            go = __all_sync(0xffffffffu, mbar_test(&ctl->pready, it & 1) && mbar_test(&ctl->ufull[uv], phv));
          }
          if (go) {
            tc_fence_after();
            if (leader) {
              const uint32_t a = v_lo + uv * (C::kUnitBytes / 16);
#pragma unroll
              for (int kk = 0; kk < kTok8 / 32; ++kk)
                mma8(tmem + C::kColO, a + kk * (2 * D), v_hi, p_lo + kk * 32, p_hi, idesc_pv, pi > 0 || kk > 0);
              tc_commit(&ctl->uempty[uv]);
              tc_commit(&ctl->pfree);
            }
            __syncwarp();
            step(uv, phv);
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
    const int key = tid;                                     // TMEM lane: key of a tile, head dim of the output
    const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
    auto wait = [&](uint64_t* bar, uint32_t parity) { wait8(bar, parity, &ctl->abort, p.status); };
    // Q: SOFT / NQ threads per row, kE values each
    constexpr int TPR = SOFT / NQ, kE = D / TPR, kQL = kE / 4;
    const int q_row = tid / TPR, q_part = tid % TPR;
    uint2 q_raw[kQL];
    int q_pos = 0;  // (window) position of row tid
    auto q_load = [&](const Seg8& s) {
      const int rg = s.row0 + q_row, h = s.kvh * p.G + rg / p.T_q, t = rg % p.T_q;
      const __nv_bfloat16* src = p.Q + s.b * p.q_sb + h * p.q_sh + t * p.q_st + q_part * kE;
#pragma unroll
      for (int i = 0; i < kQL; ++i)
        q_raw[i] = q_row < s.nrows ? *reinterpret_cast<const uint2*>(src + i * 4) : make_uint2(0, 0);
    };
    auto q_store = [&]() {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 2 * kQL; ++i) {
        const uint32_t w = i & 1 ? q_raw[i / 2].y : q_raw[i / 2].x, a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
        if (a < 0x7f80u) top = max(top, a);
        if (b < 0x7f80u) top = max(top, b);
      }
#pragma unroll
      for (int o = TPR / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      // smallest eq with |q| <= 448 * 2^eq
      const int eq = max(-100, min(119, (int)(top >> 7) - 127 - 8 + ((top & 127u) > 96u ? 1 : 0)));
      const float inv = pow2_8(-eq);
#pragma unroll
      for (int i = 0; i < kE / 4; ++i) {
        uint32_t term[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t two = k ? q_raw[i].y : q_raw[i].x;
          float2 v = make_float2(__uint_as_float(two << 16) * inv, __uint_as_float(two & 0xffff0000u) * inv);
          // (an infinite or NaN query makes its scores NaN)
          if ((two & 0x7f80u) == 0x7f80u) v.x = __int_as_float(0x7fffffff);
          if ((two & 0x7f800000u) == 0x7f800000u) v.y = __int_as_float(0x7fffffff);
          const uint32_t c = __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
          const __half2_raw hr = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
          const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hr));
          term[0] |= c << (16 * k);
          term[1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v.x - back.x, v.y - back.y), __NV_SATFINITE, __NV_E4M3)
                     << (16 * k);
        }
        // operand row nn, 16-byte piece c at nn * D + ((c ^ swizzle(nn)) * 16); the lo rows follow the hi rows
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int nn = q_row + k * NQ, sw = D == 128 ? (nn & 7) : ((nn >> 1) & 3), byte = q_part * kE + i * 4;
          *reinterpret_cast<uint32_t*>(q_s + nn * D + (((byte >> 4) ^ sw) << 4) + (byte & 15)) = term[k];
        }
      }
      if (q_part == 0) {
        ctl->qf[q_row] = pow2_8(eq) * p.scale_log2;
        ctl->nm[q_row] = 0.f;
      }
      if constexpr (WIN) {
        if (tid < NQ) ctl->pos[tid] = q_pos;
      }
      fence_proxy_async();
      mbar_arrive(&ctl->qfull);
    };

    // Scale bytes of this thread's key, fetched a tile ahead (and its page id two tiles ahead).  Small
    // pages: the key's place in its page is the same in every tile.
    const bool paged = p.kv.page_table != nullptr, small = p.kv.page_shift >= 0;
    const int page_tiles = p.kv.page_tiles;
    uint32_t ah_id = ~0u, ah_inner = 0; // page (dense: request) of the key of the tile after next, as loaded
    int ah_page = 0, ah_sub = 0;        // large pages: page of that tile, its tile within the page
    uint32_t ah_ek = 127, ah_ev = 127;  // bytes of the next tile's key
    const int32_t* ah_table = nullptr;  // the request's row of the page table
    const uint8_t *ah_ks = nullptr, *ah_vs = nullptr;  // the kv-head's scale bytes
    Win8 w = {};                        // (window) the segment's
    auto ah_look = [&](int t, int t1, int len, uint32_t b) {
      ah_id = ~0u;
      if (WIN) {
        if (t < t1 && t * kTok8 + key < len) {
          int inner = win_token8(w, t * kTok8 + key);
          ah_id = paged ? (uint32_t)page8(p.kv, (int)b, &inner) : b;
          ah_inner = inner;
        }
        return;
      }
      if (t < t1 && t * kTok8 + key < len) {
        if (!paged) {
          ah_id = b;
          ah_inner = t * kTok8 + key;
        } else {
          const int tok = t * kTok8 + key;
          ah_inner = small ? tok & (p.kv.page_size - 1) : ah_sub * kTok8 + key;
          ah_id = (uint32_t)ah_table[small ? tok >> p.kv.page_shift : ah_page];
        }
      }
      if (++ah_sub == page_tiles) {
        ah_sub = 0;
        ++ah_page;
      }
    };
    auto ah_fetch = [&]() {
      ah_ek = ah_ev = 127;   // (a key that is not there, or in a page outside the pool: value 0)
      if (ah_id < (uint32_t)p.kv.n_outer) {
        ah_ek = ah_ks[(uint64_t)ah_id * (uint64_t)p.kv.ks_sb + (uint64_t)ah_inner * (uint64_t)p.kv.ks_st];
        ah_ev = ah_vs[(uint64_t)ah_id * (uint64_t)p.kv.vs_sb + (uint64_t)ah_inner * (uint64_t)p.kv.vs_st];
      }
    };
    auto seg_fetch = [&](const Seg8& s) {
      ah_page = page_tiles == 1 ? s.t0 : s.t0 / page_tiles;
      ah_sub = s.t0 - ah_page * page_tiles;
      ah_ks = p.kv.Ks + s.kvh * p.kv.ks_sh;
      ah_vs = p.kv.Vs + s.kvh * p.kv.vs_sh;
      if (paged) ah_table = p.kv.page_table + (int64_t)s.b * p.kv.pages_per_req;
      if (WIN) {  // (rows that do not exist see what the first query sees)
        w = win8(p, s.b);
        if (tid < NQ) q_pos = w.first + (tid < s.nrows ? depth8(p, s.b, (s.row0 + tid) % p.T_q) : 0);
      }
      ah_look(s.t0, s.t1, s.len, s.b);
      q_load(s);
    };
    if (ctl->has[0]) seg_fetch(ctl->seg[0]);
    int it = 0;
    for (int k_seg = 0; ctl->has[k_seg & 1]; ++k_seg) {
      const Seg8& g = ctl->seg[k_seg & 1];
      const int t0 = g.t0, t1 = g.t1, len = g.len, b = g.b;
      if (tid == 0) {  // the next segment, read by everybody after this one's tiles
        Seg8 s = g;
        ctl->has[(k_seg + 1) & 1] = seg_next(share, &s);
        ctl->seg[(k_seg + 1) & 1] = s;
      }
      q_store();
      ah_fetch();    // (its page id has arrived by now)
      ah_look(t0 + 1, t1, len, b);
      bar8<SOFT>();  // (factors and references)
      bool unset = false;  // (window; thread r < NR) row r has no reference yet
      float2 lsum[NR / 2];
#pragma unroll
      for (int r = 0; r < NR / 2; ++r) lsum[r] = make_float2(0.f, 0.f);
      for (int t = t0; t < t1; ++t, ++it) {
        // (put into the format's range here, not where they are loaded: that would wait for them)
        const uint32_t ek = byte8(ah_ek), ev = byte8(ah_ev);
        const float kf = scale8(ek), evf = (float)(int)ev - 127.f, vinv = scale8(254u - ev);
        ah_fetch();
        ah_look(t + 2, t1, len, b);
        const int n_valid = min(kTok8, len - t * kTok8);
        const bool key_ok = key < n_valid, first = t == t0;
        const bool masked = WIN && !win_plain8(p, w, t);
        const int tok = WIN ? win_token8(w, t * kTok8 + key) : 0;
        wait(&ctl->sfull[it & 1], (it >> 1) & 1);
        tc_fence_after();
        unsigned dead = 0;  // (window) keys of this warp that no query sees
        if (WIN) {
          if (masked) dead = __ballot_sync(0xffffffffu, !win_any8(p, w, tok));
        } else if (n_valid < kTok8) {
          // tokens past the length may hold anything; their weights are 0, so V must be finite there
          const int jv = 2 * it + 1;
          wait(&ctl->ufull[jv % UNITS], (jv / UNITS) & 1);
          uint4* v = reinterpret_cast<uint4*>(smem + (jv % UNITS) * C::kUnitBytes);
#pragma unroll 1
          for (int i = n_valid * (D / 16) + tid; i < kTok8 * (D / 16); i += SOFT) v[i] = make_uint4(0, 0, 0, 0);
        }
        // x[r] = s2 + ev - M + bias (in the segment's first tile s2 + ev)
        float2 x[NR / 2];
        {
          // 8 rows at a time, hi and lo; the factors are formed while the scores are on their way
          const float2 kf2 = make_float2(kf, kf), ev2 = make_float2(evf, evf);
          const uint32_t t_s = tmem + lane_off + (it & 1) * NS;
          uint32_t raw[16];
          auto load = [&](int r0) {
            if (NQ == 8) {
              tmem_ld<16>(t_s, raw);
            } else {
              tmem_ld<8>(t_s + r0, raw);
              tmem_ld<8>(t_s + NQ + r0, raw + 8);
            }
          };
          load(0);
#pragma unroll
          for (int r0 = 0; r0 < NR; r0 += 8) {
            float2 f[4], e[4];
#pragma unroll
            for (int r = 0; r < 8; r += 4) {
              const float4 qf = *reinterpret_cast<const float4*>(&ctl->qf[r0 + r]);
              const float4 nm = *reinterpret_cast<const float4*>(&ctl->nm[r0 + r]);
              f[r / 2] = __fmul2_rn(make_float2(qf.x, qf.y), kf2);
              f[r / 2 + 1] = __fmul2_rn(make_float2(qf.z, qf.w), kf2);
              e[r / 2] = __fadd2_rn(make_float2(nm.x, nm.y), ev2);
              e[r / 2 + 1] = __fadd2_rn(make_float2(nm.z, nm.w), ev2);
            }
            tc_wait_ld();
#pragma unroll
            for (int r = 0; r < 8; r += 2) {
              const float2 sc = __fadd2_rn(make_float2(__uint_as_float(raw[r]), __uint_as_float(raw[r + 1])),
                                           make_float2(__uint_as_float(raw[8 + r]), __uint_as_float(raw[9 + r])));
              x[(r0 + r) / 2] = __ffma2_rn(sc, f[r / 2], e[r / 2]);
            }
            if (r0 + 8 < NR) load(r0 + 8);
          }
        }
        if (WIN) {
          if (masked) {
            __syncwarp();
            const uint32_t reach = win_reach8(p, w, tok);
            if (p.T_q == 1) {
              const bool ok = win_sees8(w.first, tok, reach);
#pragma unroll
              for (int r = 0; r < NR / 2; ++r)
                if (!ok) x[r] = make_float2(-INFINITY, -INFINITY);
            } else if constexpr (WIN) {
#pragma unroll
              for (int r = 0; r < NR; r += 4) {
                const int4 pos = *reinterpret_cast<const int4*>(&ctl->pos[r]);
                if (!win_sees8(pos.x, tok, reach)) x[r / 2].x = -INFINITY;
                if (!win_sees8(pos.y, tok, reach)) x[r / 2].y = -INFINITY;
                if (!win_sees8(pos.z, tok, reach)) x[r / 2 + 1].x = -INFINITY;
                if (!win_sees8(pos.w, tok, reach)) x[r / 2 + 1].y = -INFINITY;
              }
            }
          }
        } else if (n_valid < kTok8) {
          __syncwarp();  // (kept a branch: as selects it costs every tile an instruction per score)
#pragma unroll
          for (int r = 0; r < NR / 2; ++r)
            if (!key_ok) x[r] = make_float2(-INFINITY, -INFINITY);
        }
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < NR / 2; ++r) mx = max3_f(mx, x[r].x, x[r].y);
        bool missing = false;  // some row has no reference: it has seen nothing so far
        if constexpr (WIN) missing = ctl->unset;
        if ((WIN && first) || bar_or8<SOFT>(first || mx > kOver || missing)) {
          // ---- set the references to the exact maxima; later in a segment (rare) raise them, which
          // rescales O^T and the row sums ----
          if constexpr (WIN) {
            const float mine = rows_max<NQ, NR>(x);  // of row lane / (32 / NQ)
            if (lane % (32 / NQ) == 0) ctl->smax[warp][lane / (32 / NQ)] = mine;
          } else {
            float mine = -INFINITY;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              const float m = redux_max(r & 1 ? x[r / 2].y : x[r / 2].x);
              if (lane == r) mine = m;
            }
            if (lane < NR) ctl->smax[warp][lane] = mine;
          }
          bar8<SOFT>();
          if (tid < NR) {  // M rises by this much (in the first tile, from 0 to the maximum - bias)
            const float top = fmaxf(fmaxf(ctl->smax[0][tid], ctl->smax[1][tid]), fmaxf(ctl->smax[2][tid], ctl->smax[3][tid]));
            float up = first ? top - kBias : fmaxf(0.f, top - kBias);
            if (WIN) {
              const bool none = top == -INFINITY;
              if (first || unset) up = none ? 0.f : top - kBias;
              unset = (first || unset) && none && tid < g.nrows;
            }
            ctl->up[tid] = up;
            ctl->nm[tid] -= up;
          }
          if constexpr (WIN) {
            if (warp == 0) {
              const bool any = __any_sync(0xffffffffu, unset);
              if (lane == 0) ctl->unset = any;
            }
          }
          bar8<SOFT>();
          if (!first) {
            wait(&ctl->pfree, (it - 1) & 1);  // the output MMAs of the tile before have retired
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < 3; ++k) {     // the three terms' accumulators
#pragma unroll 1
              for (int r = 0; r < NR; r += 8) {
                uint32_t o[8];
                const uint32_t at = tmem + lane_off + C::kColO + k * NR + r;
                tmem_ld<8>(at, o);
                tc_wait_ld();
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                  const float a = __uint_as_float(o[c]);
                  // (window: 0 stays 0, a first reference far below 0 makes the factor infinite)
                  o[c] = WIN && a == 0.f ? 0u : __float_as_uint(a * ex2_ftz(-ctl->up[r + c]));
                }
                tmem_st8(at, o);
              }
            }
            tc_wait_st();
          }
#pragma unroll
          for (int r = 0; r < NR / 2; ++r) {
            const float2 up = *reinterpret_cast<const float2*>(&ctl->up[2 * r]);
            x[r] = __fadd2_rn(x[r], make_float2(-up.x, -up.y));
            if (!first) {
              float2 f = make_float2(ex2_ftz(-up.x), ex2_ftz(-up.y));
              if (WIN && lsum[r].x == 0.f) f.x = 0.f;
              if (WIN && lsum[r].y == 0.f) f.y = 0.f;
              lsum[r] = __fmul2_rn(lsum[r], f);
            }
          }
        }
        {
          // columns term * NR + row, 16 to a 16-byte piece per key, in words of 4; nothing behind them.
          // All are formed before the wait: the output MMAs of the tile before run meanwhile (16 rows at
          // a time behind it: 64 rows, 16 x 16384 tokens, 178 us against 174).
          const float2 vinv2 = make_float2(vinv, vinv);
          constexpr int W = NR / 4;
          uint32_t word[NP / 4] = {};
#pragma unroll
          for (int q = 0; q < W; ++q) {
            uint32_t w[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int i = 2 * q + k;
              const float2 e = make_float2(ex2_ftz(x[i].x), ex2_ftz(x[i].y));
              lsum[i] = __ffma2_rn(e, vinv2, lsum[i]);
              w[k] = h2_bits(__float22half2_rn(e));
            }
            const uint32_t a1 = residue(w[0]), b1 = residue(w[1]);
            word[q] = __byte_perm(w[0], w[1], 0x7531);
            word[W + q] = __byte_perm(a1, b1, 0x7531);
            // (the last term rounds)
            word[2 * W + q] = __byte_perm(residue(a1) + 0x00800080u, residue(b1) + 0x00800080u, 0x7531);
          }
          if (!first) wait(&ctl->pfree, (it - 1) & 1);  // P^T has been consumed
#pragma unroll
          for (int k = 0; k < NP / 16; ++k)
            *reinterpret_cast<uint4*>(p_s + k * (kTok8 * 16) + key * 16) =
                make_uint4(word[4 * k], word[4 * k + 1], word[4 * k + 2], word[4 * k + 3]);
          if (WIN && dead) {  // such tokens may hold anything; their weights are 0, so V must be finite there
            const int jv = 2 * it + 1;
            wait(&ctl->ufull[jv % UNITS], (jv / UNITS) & 1);
            constexpr int kPieces = D / 16;  // 16-byte pieces of a row
            uint8_t* v = smem + (jv % UNITS) * C::kUnitBytes + warp * 32 * D + (lane % kPieces) * 16;
#pragma unroll 1
            for (int r = lane / kPieces; r < 32; r += 32 / kPieces)
              if (dead >> r & 1) *reinterpret_cast<uint4*>(v + r * D) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
          tc_fence_before();
        }
        mbar_arrive(&ctl->pready);
      }

      // ---- the segment's end: what the next one needs is fetched first ----
      const Seg8& done = g;
      if (ctl->has[(k_seg + 1) & 1]) seg_fetch(ctl->seg[(k_seg + 1) & 1]);
      // row sums: halve the rows a lane holds at every step, lane / (32 / NQ) is the row in the end
      {
        float v[NQ];
#pragma unroll
        for (int r = 0; r < NQ; ++r) v[r] = r >= NR ? 0.f : (r & 1) ? lsum[r / 2].y : lsum[r / 2].x;
        int n = NQ;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
          if (n > 1) {
            n /= 2;
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < NQ / 2; ++i) {
              if (i < n) {
                const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
              }
            }
          } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
          }
        }
        if (CL) {
          wait(&ctl->pfree, (it - 1) & 1);
          tc_fence_after();
          parts.ready();
          if (lane % (32 / NQ) == 0) parts.put_l(lane / (32 / NQ), warp, v[0]);
          if (tid < NQ) parts.put_m(tid, -ctl->nm[tid]);
#pragma unroll 1
          for (int q = 0; q < NR && q < done.nrows; q += 8) {
            uint32_t o[3][8];
#pragma unroll
            for (int k = 0; k < 3; ++k) tmem_ld<8>(tmem + lane_off + C::kColO + k * NR + q, o[k]);
            tc_wait_ld();
#pragma unroll
            for (int c = 0; c < 8; ++c)
              if (key < D)
                parts.put_a(q + c, key, fmaf(__uint_as_float(o[2][c]), 1.f / 64.f,
                                             fmaf(__uint_as_float(o[1][c]), 0.125f, __uint_as_float(o[0][c]))));
          }
          break;
        }
        bar8<SOFT>();  // (every thread is done with smax as maxima)
        if (lane % (32 / NQ) == 0) ctl->smax[warp][lane / (32 / NQ)] = v[0];
      }
      wait(&ctl->pfree, (it - 1) & 1);
      tc_fence_after();
      bar8<SOFT>();
      // the unit's result when it is whole, this CTA's state of it when it is cut
      const bool whole = done.t0 == 0 && done.t1 == done.n;
      float* slot = slot8(p, share, done.start, share.idx);
      if (tid < done.nrows) {
        // (the sums are of 2^(s2 - M + bias))
        const float m = -ctl->nm[tid], l = (ctl->smax[0][tid] + ctl->smax[1][tid]) + (ctl->smax[2][tid] + ctl->smax[3][tid]);
        if (whole) put_ml8(p, done, tid, m, l);
        else reinterpret_cast<float2*>(slot)[tid] = make_float2(m, l);
        if (!whole && done.t0 == 0 && !p.O) put_cut8(p, share, done, tid);
        ctl->up[tid] = l > 0.f || l != l ? 1.f / l : 0.f;
      }
      if constexpr (WIN) {
        if (tid == 0) ctl->unset = 0;
      }
      bar8<SOFT>();
      const int64_t pair = (int64_t)done.b * p.H_kv + done.kvh;
      const bool to_o = whole && p.O;
      __nv_bfloat16* o_row = p.O + (pair * p.R + done.row0) * D + key;
      float* a_row = (whole ? p.part_a + (pair * p.R_stride + done.row0) * D : slot + 4 * p.rows_per_tile) + key;
#pragma unroll 1
      for (int q = 0; q < NR && q < done.nrows; q += 8) {
        uint32_t o[3][8];
#pragma unroll
        for (int k = 0; k < 3; ++k) tmem_ld<8>(tmem + lane_off + C::kColO + k * NR + q, o[k]);
        tc_wait_ld();
        const int n = key < D ? done.nrows - q : 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float a = fmaf(__uint_as_float(o[2][c]), 1.f / 64.f,
                               fmaf(__uint_as_float(o[1][c]), 0.125f, __uint_as_float(o[0][c])));
          if (c < n) {
            if (to_o) {
              o_row[(q + c) * D] = __float2bfloat16_rn(a * ctl->up[q + c]);
            } else {
              a_row[(q + c) * D] = a;
            }
          }
        }
      }
      tc_fence_before();
      bar8<SOFT>();  // sums, references and Q may be written anew
    }
    if (CL) {
      if (!ctl->has[0]) {
        parts.ready();
        parts.put_none(tid);
      }
    } else if ((int)blockIdx.x < p.B) {
      put_empty8<WIN>(p, tid, SOFT);
    }
  }

  tc_fence_before();
  if (!CL) {
    __syncthreads();
  } else {
    if (warp >= 4) parts.ready();
    parts.end(p, place);
  }
  if (warp == kTmemWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
}

template <int NR, int D, bool WIN, bool CL>
cudaError_t prepare8() {
  return cudaFuncSetAttribute(attn8_tc_kernel<NR, D, WIN, CL>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              Cfg8<NR, D, WIN>::kSmem);
}
template <int NR, int D, bool WIN>
cudaError_t launch8(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  using C = Cfg8<NR, D, WIN>;
  if constexpr (WIN) {
    if (p.mode == kCluster8)
      return launch_kernel_cluster(attn8_tc_kernel<NR, D, true, true>,
                                   dim3((unsigned)p.B * p.H_kv * p.row_tiles * p.cluster), dim3(C::kThreads), C::kSmem, s,
                                   pdl, (unsigned)p.cluster, p, tmK, tmV);
  }
  return launch_kernel(attn8_tc_kernel<NR, D, WIN, false>, dim3(p.shares * p.row_tiles), dim3(C::kThreads), C::kSmem, s, pdl,
                       p, tmK, tmV);
}
template <int D, bool WIN, bool CL>
cudaError_t prepare_rows() {
  cudaError_t e = prepare8<8, D, WIN, CL>();
  if (e == cudaSuccess) e = prepare8<16, D, WIN, CL>();
  if (e == cudaSuccess) e = prepare8<24, D, WIN, CL>();
  if (e == cudaSuccess) e = prepare8<32, D, WIN, CL>();
  return e;
}
template <int D, bool WIN>
cudaError_t launch_rows(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  // (24 rows as 32: 247 us against 242 for 8 x 98304 tokens; 40 rows as 2 x 32 against 2 x 24: 172 and 155)
  if (p.rows_per_tile <= 8) return launch8<8, D, WIN>(p, tmK, tmV, s, pdl);
  if (p.rows_per_tile <= 16) return launch8<16, D, WIN>(p, tmK, tmV, s, pdl);
  if (p.rows_per_tile <= 24) return launch8<24, D, WIN>(p, tmK, tmV, s, pdl);
  return launch8<32, D, WIN>(p, tmK, tmV, s, pdl);
}

}  // namespace

cudaError_t attn8_tc_prepare() {
  cudaError_t e = prepare_rows<128, false, false>();
  if (e == cudaSuccess) e = prepare_rows<64, false, false>();
  if (e == cudaSuccess) e = prepare_rows<128, true, false>();
  if (e == cudaSuccess) e = prepare_rows<64, true, false>();
  if (e == cudaSuccess) e = prepare_rows<128, true, true>();
  if (e == cudaSuccess) e = prepare_rows<64, true, true>();
  return e;
}

cudaError_t launch_attn8_tc(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  if (p.window) return p.d == 128 ? launch_rows<128, true>(p, tmK, tmV, s, pdl) : launch_rows<64, true>(p, tmK, tmV, s, pdl);
  return p.d == 128 ? launch_rows<128, false>(p, tmK, tmV, s, pdl) : launch_rows<64, false>(p, tmK, tmV, s, pdl);
}

}  // namespace ss
