// Attention over a window of a bf16 cache on the tensor cores: decoding steps, pieces of a prompt, and chunks of a
// round (span8 in kv8.cuh says which tokens are walked and how they are numbered).
//
//   S^T = K Q^T    M = 128 keys of the tile, N = rows (16 at least), K = d    (d / 16 steps)
//   O^T = V^T P^T  M = 128 head dims,        N = rows x terms, K = 128 keys   (8 steps)
//
// A CTA walks its share of the tiles (kv8.cuh) like the 8-bit kernel: a TMA producer warp that gathers tiles granule
// by granule and runs ahead across segment ends, an MMA issuer warp, 4 softmax warps whose thread is a key of the
// tile in the scores and a head dim in the output; references M raised lazily (exact maximum of the first tile,
// later when a score exceeds M by 16 in base 2), row sums in fp32 from unrounded weights.  Weights go to the output
// MMA as two bf16 terms side by side on the N axis (off by 2^-16), where shared memory has room for them: with up
// to 8 rows the second term takes the columns that N = 16 leaves idle; 17 to 32 rows at head dim 128 take one term
// (off by 2^-8 at most, as in the chunk kernels), or the ring would lose one of its three units.  In units of 16 rows, which
// have two terms, such calls read K and V twice: 64 kv-heads of 32 rows over 4000 tokens 26.4 us against 33.0.  (Outputs are
// off by 1.66e-3 in the 2-norm, their rounding to bf16; with one term by 1.69e-3 where many tokens weigh, up to 2.2e-3 where
// a few do.)
//
// Masks.  All rows see all of a tile but in the few tiles at the window's ends, the sinks' end and among the queries
// themselves (win_plain8); there a score that its row does not see becomes -inf, by key where the request has one
// query, else by row and key.  V rows that no query sees may hold anything and are cleared in the staged tile (their
// weight is 0, but 0 * NaN is not).  A row that sees nothing of a segment's first tiles has no reference yet: the
// next tiles take the raising path until it has one.
// Every wait is bounded; on expiry the CTA raises SS_DEV_WAIT_EXPIRED and returns.
#include "kv8_tc.cuh"

namespace ss {
namespace {

using namespace ss::tc;

constexpr float kOver = 16.f;
constexpr int kBox = kTok8 * 128;  // 64 head dims of a tile's tokens

template <int NR>
struct alignas(16) CtlW {
  uint64_t ufull[8], uempty[8];
  uint64_t sfull[2], pready, pfree, qfull, segfull;
  uint32_t tmem_base;
  volatile uint32_t abort;
  // The current and the next segment, in use by turns.  The MMA warp writes the next one's slot behind a segment's first
  // scores, that is once all softmax threads have arrived on qfull for that segment: from their arrival for segment k + 1
  // on they read nothing of segment k's slot.
  int has[2];
  int unset;                      // rows without a reference
  int go;                         // a segment follows
  Seg8 seg[2];
  Win8 win[2];
  Share8 share;
  alignas(16) float nm[NR];       // -M
  alignas(16) float up[NR];       // rise of the references; at a segment's end 1 / row sum
  alignas(16) int pos[NR];        // the rows' positions
};

// NR = rows, D = head dim.
template <int NR, int D>
struct CfgW {
  static constexpr int kSoft = 128, kThreads = kSoft + 64;  // softmax threads, all threads
  static constexpr int kHalves = D / 64;
  static constexpr int kUnitBytes = kHalves * kBox;         // one K or V tile
  static constexpr int NQ = NR < 16 ? 16 : NR;              // N is a multiple of 16
  static constexpr int kTerms = NR == 32 && D == 128 ? 1 : 2;
  static constexpr int NP = kTerms * NR;
  static constexpr int kQHalf = NQ * 128;
  static constexpr int kQBytes = kHalves * kQHalf;
  static constexpr int kPBytes = kTok8 * NP * 2;
  static constexpr int kCtlBytes = (sizeof(CtlW<NR>) + 127) / 128 * 128;
  static constexpr int kPartsBytes = Parts8<NR, D, NR == 8>::kBytes;   // (clusters)
  static constexpr int kRest = (kQBytes + 1023) / 1024 * 1024 + kPBytes + kCtlBytes + kPartsBytes;
  // head dim 64: the output MMA's upper 64 rows read one box further on (results never used), the last
  // unit's inside this window too
  static constexpr int kAfter = D == 64 && kRest < kBox ? kBox : kRest;
  static constexpr int kPerSM = 2;
  static constexpr int kUnits0 = (113 * 1024 - kAfter) / kUnitBytes;
  static constexpr int kUnits = kUnits0 > 8 ? 8 : kUnits0;
  static constexpr int kOffQ = kUnits * kUnitBytes;
  static constexpr int kOffP = kOffQ + (kQBytes + 1023) / 1024 * 1024;
  static constexpr int kOffCtl = kOffP + kPBytes;
  static constexpr int kOffParts = kOffCtl + kCtlBytes;
  static constexpr int kSmem = kOffQ + kAfter;
  static constexpr uint32_t kColO = 2 * NQ;                 // two score buffers, then O^T
  static constexpr int kCols = 2 * NQ + NP;
  static constexpr uint32_t kTmemCols = kCols <= 64 ? 64 : 128;
  static_assert(kUnits >= 3 && kCols <= 128 && kPBytes >= 4 * NR * 4 && kUnits * kUnitBytes >= NR * (D + 5) * 4, "shape");
};

// Two bf16 values, infinities made NaN: an infinite query's scores might all be -inf, and its row look empty.
__device__ __forceinline__ uint32_t nan_of(uint32_t two) {
  if ((two & 0x7f80u) == 0x7f80u) two |= 0x7fffu;
  if ((two & 0x7f800000u) == 0x7f800000u) two |= 0x7fff0000u;
  return two;
}

// CL: a unit is one cluster's (kCluster8), each CTA has one segment.
template <int NR, int D, bool CL>
__global__ void __launch_bounds__(CfgW<NR, D>::kThreads, CfgW<NR, D>::kPerSM)
window_tc_kernel(const __grid_constant__ Attn8Params p, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV) {
  using C = CfgW<NR, D>;
  constexpr int UNITS = C::kUnits, NQ = C::NQ, SOFT = C::kSoft;
  extern __shared__ __align__(1024) uint8_t smem[];
  CtlW<NR>* ctl = reinterpret_cast<CtlW<NR>*>(smem + C::kOffCtl);
  uint8_t* q_s = smem + C::kOffQ;
  uint8_t* p_s = smem + C::kOffP;
  float* smax = reinterpret_cast<float*>(p_s);    // [4][NR] maxima and sums of the warps, while P is not in use
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
      mbar_init(&ctl->pready, SOFT);
      mbar_init(&ctl->pfree, 1);
      mbar_init(&ctl->qfull, SOFT);
      mbar_init(&ctl->segfull, 1);
      ctl->abort = 0;
      ctl->unset = 0;
      fence_barrier_init();
    }
    __syncwarp();
    // The others wait for this below; the producer goes on: its first copies have a chain of dependent loads in
    // front of them (length, page id, K) that all the rest waits for.
    __threadfence_block();
    asm volatile("barrier.cta.arrive 2, %0;" ::"n"(C::kThreads) : "memory");
  }
  Place8 place = {};
  if (CL) place = cluster_place8(p);
  using P = Parts8<NR, D, CL && NR == 8>;
  const P parts(reinterpret_cast<float*>(smem + (NR == 8 ? C::kOffParts : 0)), p, place);
  auto find = [&]() {
    Share8 s = {};
    if (!CL) s = find_share8<true>(p);
    return s;
  };
  auto seg_first = [&](const Share8& s, Seg8* g) { return CL ? cluster_seg8(p, place, g) : seg_first8<true>(p, s, g); };
  auto seg_next = [&](const Share8& s, Seg8* g) { return !CL && seg_next8<true>(p, s, g); };
  // (tensor memory is taken after the wait: the kernel in front may still be about to allocate its own)
  pdl_wait_prior();
  pdl_launch_dependents();
  if (warp != kProducerWarp) {
    if (warp == kMmaWarp) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                   "r"(C::kTmemCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 0) {
      const Share8 share = find();
      if (lane == 0) {
        ctl->share = share;
        const bool some = seg_first(share, &ctl->seg[0]);
        ctl->has[0] = some;
        if (some) ctl->win[0] = win8(p, ctl->seg[0].b);
      }
    }
    tc_fence_before();
    asm volatile("barrier.cta.sync 2, %0;" ::"n"(C::kThreads) : "memory");
    tc_fence_after();
  }
  const uint32_t tmem = ctl->tmem_base;  // (not for the producer, as the share)
  const Share8& share = ctl->share;
  auto mwait = [&](uint64_t* bar, uint32_t parity) {
    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, &ctl->abort, p.status);
  };

  if (warp == kProducerWarp) {
    // ===== TMA producer: a lane brings one granule's 64 head dims of every tile =====
    const uint64_t pol = p.row_tiles > 1 ? l2_evict_normal_policy() : l2_evict_first_policy();
    const int gl = p.gran_log2, sub = lane / C::kHalves, half = lane % C::kHalves;
    const bool mine = sub < kTok8 >> gl;
    const uint32_t at = smem_u32(smem) + half * kBox + (sub << gl) * 128;
    int j = 0, u = 0;      // units filled so far, the next one's place in the ring
    uint32_t ph = 1;       // parity of its release
    bool ok = true;
    const Share8 share = find();
    Seg8 g;
    for (bool more = seg_first(share, &g); more && ok; more = seg_next(share, &g)) {
      const Win8 w = win8(p, g.b);
      int inner = 0, outer = 0;
      auto look = [&](int t) {  // this lane's granule of tile t
        const int v = t * kTok8 + (sub << gl);
        outer = p.kv.n_outer;   // outside the tensor: reads as zeros
        inner = 0;
        if (!mine || t >= g.t1 || v >= g.len) return;
        inner = win_token8(w, v);
        int id = g.b;
        if (p.kv.page_table) id = page8(p.kv, g.b, &inner);
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
          if (mine) {
            if (kv) tma_load_4d(at + u * C::kUnitBytes, &tmV, half * 64, inner, g.kvh, outer, &ctl->ufull[u], pol);
            else tma_load_4d(at + u * C::kUnitBytes, &tmK, half * 64, inner, g.kvh, outer, &ctl->ufull[u], pol);
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
    __syncwarp();
    if (p.depth) check_depths8(p);
  } else if (warp == kMmaWarp) {
    // ===== MMA issuer: polls for whichever of its two next operations can go =====
    constexpr uint32_t idesc_qk = make_idesc_major(128, NQ, false, false), idesc_pv = make_idesc_major(128, C::NP, true, true);
    const bool leader = elect_one();
    const uint32_t base = smem_u32(smem), q_addr = smem_u32(q_s), p_addr = smem_u32(p_s);
    int it0 = 0, seg = 0;  // tiles and segments before this one
    bool ok = true;
    Seg8 g = ctl->seg[0];
    for (bool more = ctl->has[0]; more && ok; ++seg) {
      const int n = g.t1 - g.t0;
      int qi = 0, pi = 0;
      bool q_there = false;
      unsigned long long t0 = gtime_ns();
      uint32_t spins = 0;
      while (pi < n) {
        bool did = false;
        if (qi < n && qi < pi + 2) {
          const int it = it0 + qi, jk = 2 * it, u = jk % UNITS;
          if (!q_there) q_there = __all_sync(0xffffffffu, mbar_test(&ctl->qfull, seg & 1));
          if (q_there && __all_sync(0xffffffffu, mbar_test(&ctl->ufull[u], (jk / UNITS) & 1))) {
            tc_fence_after();
            if (leader) {
              const uint32_t k_addr = base + u * C::kUnitBytes;
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk)
                mma_ss(tmem + (it & 1) * NQ, desc_kmajor(k_addr + (kk >> 2) * kBox + (kk & 3) * 32),
                       desc_kmajor(q_addr + (kk >> 2) * C::kQHalf + (kk & 3) * 32), idesc_qk, kk > 0);
              tc_commit(&ctl->uempty[u]);
              tc_commit(&ctl->sfull[it & 1]);
            }
            __syncwarp();
            if (!CL && qi == 0) {  // the next segment, while the softmax warps are at the first tile, their longest
              more = seg_next(share, &g);
              if (lane == 0) {
                ctl->seg[(seg + 1) & 1] = g;
                ctl->has[(seg + 1) & 1] = more;
                if (more) ctl->win[(seg + 1) & 1] = win8(p, g.b);
                mbar_arrive(&ctl->segfull);
              }
              __syncwarp();
            }
            ++qi;
            did = true;
          }
        }
        if (pi < qi) {
          const int it = it0 + pi, jv = 2 * it + 1, u = jv % UNITS;
          // with the scores two tiles ahead nothing but this can go: sleep on it instead of polling
          bool go = true;
          if (qi == n || qi == pi + 2) {
            ok = mwait(&ctl->pready, it & 1) && mwait(&ctl->ufull[u], (jv / UNITS) & 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
          } else {
            go = __all_sync(0xffffffffu, mbar_test(&ctl->pready, it & 1) && mbar_test(&ctl->ufull[u], (jv / UNITS) & 1));
          }
          if (go) {
            tc_fence_after();
            if (leader) {
              const uint32_t v_addr = base + u * C::kUnitBytes;
#pragma unroll
              for (int kk = 0; kk < kTok8 / 16; ++kk)
                mma_ss(tmem + C::kColO, desc_mnmajor(v_addr + kk * 2048, kBox),
                       desc_mnmajor_plain(p_addr + kk * 256, 128, kTok8 * 16), idesc_pv, pi > 0 || kk > 0);
              tc_commit(&ctl->uempty[u]);
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
      if (CL) break;
    }
  } else {
    // ===== softmax warps =====
    const int key = tid;                                     // TMEM lane: key of a tile, head dim of the output
    const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
    auto wait = [&](uint64_t* bar, uint32_t parity) { wait8(bar, parity, &ctl->abort, p.status); };
    // Q: kQP 16-byte pieces of a row per thread, K-major operand with 128-byte swizzle, rows of zeros behind
    constexpr int kQP = NQ * (D / 8) / SOFT;
    static_assert(kQP * SOFT == NQ * (D / 8), "pieces");
    uint4 q_raw[kQP];
    int q_pos = 0;
    auto q_load = [&](const Seg8& s, int first) {
#pragma unroll
      for (int i = 0; i < kQP; ++i) {
        const int n = (tid + i * SOFT) / (D / 8), c8 = (tid + i * SOFT) % (D / 8);
        q_raw[i] = make_uint4(0, 0, 0, 0);
        if (n < s.nrows) {
          const int rg = s.row0 + n, h = s.kvh * p.G + rg / p.T_q, t = rg % p.T_q;
          q_raw[i] = *reinterpret_cast<const uint4*>(p.Q + s.b * p.q_sb + h * p.q_sh + t * p.q_st + c8 * 8);
        }
      }
      // (rows that do not exist see what the first query sees)
      if (tid < NR) q_pos = first + (tid < s.nrows ? depth8(p, s.b, (s.row0 + tid) % p.T_q) : 0);
    };
    auto q_store = [&]() {
#pragma unroll
      for (int i = 0; i < kQP; ++i) {
        const int n = (tid + i * SOFT) / (D / 8), c8 = (tid + i * SOFT) % (D / 8);
        q_raw[i] = make_uint4(nan_of(q_raw[i].x), nan_of(q_raw[i].y), nan_of(q_raw[i].z), nan_of(q_raw[i].w));
        *reinterpret_cast<uint4*>(q_s + (c8 >> 3) * C::kQHalf + n * 128 + (((c8 & 7) ^ (n & 7)) << 4)) = q_raw[i];
      }
      if (tid < NR) {
        ctl->nm[tid] = 0.f;
        ctl->pos[tid] = q_pos;
      }
      fence_proxy_async();
      mbar_arrive(&ctl->qfull);
    };
    const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
    bool go = ctl->has[0];
    if (go) {
      q_load(ctl->seg[0], ctl->win[0].first);
      q_store();
      bar8<SOFT>();  // (references and positions)
    }
    int it = 0;
    for (int k_seg = 0; go; ++k_seg) {
      const Seg8& g = ctl->seg[k_seg & 1];
      const int t0 = g.t0, t1 = g.t1;
      const Win8 w = ctl->win[k_seg & 1];
      bool unset = false;  // (thread r < NR) row r has no reference yet
      float2 lsum[NR / 2];
#pragma unroll
      for (int r = 0; r < NR / 2; ++r) lsum[r] = make_float2(0.f, 0.f);
      for (int t = t0; t < t1; ++t, ++it) {
        const bool first = t == t0, plain = win_plain8(p, w, t);
        const int tok = win_token8(w, t * kTok8 + key);
        wait(&ctl->sfull[it & 1], (it >> 1) & 1);
        tc_fence_after();
        // x[r] = s2 - M (in the segment's first tile s2)
        float2 x[NR / 2];
        {
          const uint32_t t_s = tmem + lane_off + (it & 1) * NQ;
          uint32_t raw[NR];
#pragma unroll
          for (int r0 = 0; r0 < NR; r0 += 16) tmem_ld<NR < 16 ? 8 : 16>(t_s + r0, raw + r0);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < NR; r += 4) {
            const float4 nm = *reinterpret_cast<const float4*>(&ctl->nm[r]);
            x[r / 2] = fma2_f(make_float2(__uint_as_float(raw[r]), __uint_as_float(raw[r + 1])), sc2, make_float2(nm.x, nm.y));
            x[r / 2 + 1] = fma2_f(make_float2(__uint_as_float(raw[r + 2]), __uint_as_float(raw[r + 3])), sc2, make_float2(nm.z, nm.w));
          }
        }
        unsigned dead = 0;  // keys of this warp that no query sees
        if (!plain) {
          dead = __ballot_sync(0xffffffffu, !win_any8(p, w, tok));
          const uint32_t reach = win_reach8(p, w, tok);
          if (p.T_q == 1) {
            const bool ok = win_sees8(w.first, tok, reach);
#pragma unroll
            for (int r = 0; r < NR / 2; ++r)
              if (!ok) x[r] = make_float2(-INFINITY, -INFINITY);
          } else {
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
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < NR / 2; ++r) mx = max3_f(mx, x[r].x, x[r].y);
        if (first || bar_or8<SOFT>(mx > kOver || ctl->unset)) {
          // ---- set the references to the exact maxima; later in a segment (rare) raise them, which
          // rescales O^T and the row sums ----
          if (!first) {
            wait(&ctl->pfree, (it - 1) & 1);  // the output MMAs of the tile before have retired
            tc_fence_after();
          }
          const float mine = rows_max<NR, NR>(x);  // of row lane / (32 / NR)
          if (lane % (32 / NR) == 0) smax[warp * NR + lane / (32 / NR)] = mine;
          bar8<SOFT>();
          if (warp == 0) {  // M rises by this much (from 0 to the maximum where there was none)
            if (lane < NR) {
              const float top = fmaxf(fmaxf(smax[lane], smax[NR + lane]), fmaxf(smax[2 * NR + lane], smax[3 * NR + lane]));
              const bool none = top == -INFINITY;
              const float up = first || unset ? (none ? 0.f : top) : fmaxf(0.f, top);
              unset = (first || unset) && none && lane < g.nrows;
              ctl->up[lane] = up;
              ctl->nm[lane] -= up;
            }
            const bool any = __any_sync(0xffffffffu, unset);
            if (lane == 0) ctl->unset = any;
          }
          bar8<SOFT>();
          if (!first) {
#pragma unroll 1
            for (int c = 0; c < C::NP; c += 8) {
              uint32_t o[8];
              tmem_ld<8>(tmem + lane_off + C::kColO + c, o);
              tc_wait_ld();
#pragma unroll
              for (int k = 0; k < 8; ++k) {  // (0 stays 0: a first reference far below 0 makes the factor infinite)
                const float a = __uint_as_float(o[k]);
                o[k] = a == 0.f ? 0u : __float_as_uint(a * ex2_ftz(-ctl->up[(c + k) % NR]));
              }
              tmem_st8(tmem + lane_off + C::kColO + c, o);
            }
            tc_wait_st();
          }
#pragma unroll
          for (int r = 0; r < NR / 2; ++r) {
            const float2 up = *reinterpret_cast<const float2*>(&ctl->up[2 * r]);
            x[r] = add2_f(x[r], make_float2(-up.x, -up.y));
            if (!first) {
              lsum[r].x = lsum[r].x == 0.f ? 0.f : lsum[r].x * ex2_ftz(-up.x);
              lsum[r].y = lsum[r].y == 0.f ? 0.f : lsum[r].y * ex2_ftz(-up.y);
            }
          }
        }
        {
          // 16-byte pieces: rows 8 c .. 8 c + 7 of a term
          uint32_t hi[NR / 2], lo[NR / 2];
#pragma unroll
          for (int r = 0; r < NR / 2; ++r) {
            const float2 e = make_float2(ex2_ftz(x[r].x), ex2_ftz(x[r].y));
            lsum[r] = add2_f(lsum[r], e);
            const __nv_bfloat162 h = __floats2bfloat162_rn(e.x, e.y);
            hi[r] = *reinterpret_cast<const uint32_t*>(&h);
            if (C::kTerms == 2) {
              const __nv_bfloat162 l = __floats2bfloat162_rn(e.x - __uint_as_float(hi[r] << 16), e.y - __uint_as_float(hi[r] & 0xffff0000u));
              lo[r] = *reinterpret_cast<const uint32_t*>(&l);
            }
          }
          if (!first) wait(&ctl->pfree, (it - 1) & 1);  // P^T has been consumed
#pragma unroll
          for (int c = 0; c < NR / 8; ++c) {
            *reinterpret_cast<uint4*>(p_s + c * (kTok8 * 16) + key * 16) = make_uint4(hi[4 * c], hi[4 * c + 1], hi[4 * c + 2], hi[4 * c + 3]);
            if (C::kTerms == 2)
              *reinterpret_cast<uint4*>(p_s + (NR / 8 + c) * (kTok8 * 16) + key * 16) =
                  make_uint4(lo[4 * c], lo[4 * c + 1], lo[4 * c + 2], lo[4 * c + 3]);
          }
          if (dead) {  // such tokens may hold anything; their weights are 0, so V must be finite there
            const int jv = 2 * it + 1;
            wait(&ctl->ufull[jv % UNITS], (jv / UNITS) & 1);
            constexpr int kPieces = 8 * C::kHalves;  // 16-byte pieces of a row
            const int piece = lane % kPieces;
            uint8_t* v = smem + (jv % UNITS) * C::kUnitBytes + (piece >> 3) * kBox + warp * 32 * 128 + (piece & 7) * 16;
#pragma unroll 1
            for (int r = lane / kPieces; r < 32; r += 32 / kPieces)
              if (dead >> r & 1) *reinterpret_cast<uint4*>(v + r * 128) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
          tc_fence_before();
        }
        mbar_arrive(&ctl->pready);
      }

      // ---- the segment's end: what the next one needs is fetched first ----
      const Seg8 done = g;  // (by value: its slot is the MMA warp's from q_store on)
      const int next = (k_seg + 1) & 1;
      if (!CL) {
        wait(&ctl->segfull, k_seg & 1);
        if (!ctl->abort && ctl->has[next]) q_load(ctl->seg[next], ctl->win[next].first);  // (aborted: nobody may have left one)
      }
      // row sums: halve the rows a lane holds at every step, lane / (32 / NR) is the row in the end
      float v[NR];
      {
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
      }
      wait(&ctl->pfree, (it - 1) & 1);
      tc_fence_after();
      if (CL) {
        parts.ready();
        if (lane % (32 / NR) == 0) parts.put_l(lane / (32 / NR), warp, v[0]);
        if (tid < NR) parts.put_m(tid, -ctl->nm[tid]);
#pragma unroll 1
        for (int q = 0; q < NR && q < done.nrows; q += 8) {
          uint32_t o[C::kTerms][8];
#pragma unroll
          for (int k = 0; k < C::kTerms; ++k) tmem_ld<8>(tmem + lane_off + C::kColO + k * NR + q, o[k]);
          tc_wait_ld();
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            float a = __uint_as_float(o[0][c]);
            if (C::kTerms == 2) a += __uint_as_float(o[C::kTerms - 1][c]);
            if (key < D) parts.put_a(q + c, key, a);
          }
        }
        break;
      }
      bar8<SOFT>();  // (nobody's P is in use)
      if (lane % (32 / NR) == 0) smax[warp * NR + lane / (32 / NR)] = v[0];
      bar8<SOFT>();
      // the unit's result when it is whole, this CTA's state of it when it is cut
      const bool whole = done.t0 == 0 && done.t1 == done.n;
      float* slot = slot8(p, share, done.start, share.idx);
      if (tid < done.nrows) {
        const float m = -ctl->nm[tid], l = (smax[tid] + smax[NR + tid]) + (smax[2 * NR + tid] + smax[3 * NR + tid]);
        if (whole) put_ml8(p, done, tid, m, l);
        else reinterpret_cast<float2*>(slot)[tid] = make_float2(m, l);
        if (!whole && done.t0 == 0 && !p.O) put_cut8(p, share, done, tid);
        ctl->up[tid] = l > 0.f || l != l ? 1.f / l : 0.f;
      }
      if (tid == 0) {
        ctl->unset = 0;
        ctl->go = !ctl->abort && ctl->has[next];  // (one decision for all)
      }
      bar8<SOFT>();
      go = ctl->go;
      if (go) q_store();  // the next segment's scores come while this one's output leaves (64 x 1024 tokens: 50.7 -> 48.4 us)
      const int64_t pair = (int64_t)done.b * p.H_kv + done.kvh;
      const bool to_o = whole && p.O;
      constexpr int kOut = NR < 16 ? 8 : 16;
      __nv_bfloat16* o_row = p.O + (pair * p.R + done.row0) * D + key;
      float* a_row = (whole ? p.part_a + (pair * p.R_stride + done.row0) * D : slot + 4 * p.rows_per_tile) + key;
#pragma unroll 1
      for (int q = 0; q < NR && q < done.nrows; q += kOut) {
        uint32_t o[C::kTerms][kOut];
#pragma unroll
        for (int k = 0; k < C::kTerms; ++k) tmem_ld<kOut>(tmem + lane_off + C::kColO + k * NR + q, o[k]);
        tc_wait_ld();
        const int n = key < D ? done.nrows - q : 0;
#pragma unroll
        for (int c = 0; c < kOut; ++c) {
          float a = __uint_as_float(o[0][c]);
          if (C::kTerms == 2) a += __uint_as_float(o[C::kTerms - 1][c]);
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
      put_empty8<true>(p, tid, SOFT);
    }
  }

  tc_fence_before();
  if (!CL) {
    __syncthreads();
  } else {
    if (warp >= 4) parts.ready();
    parts.end(p, place);
  }
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
}

template <int NR, int D>
cudaError_t prepare() {
  const cudaError_t e = cudaFuncSetAttribute(window_tc_kernel<NR, D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, CfgW<NR, D>::kSmem);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(window_tc_kernel<NR, D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, CfgW<NR, D>::kSmem);
}
template <int NR, int D>
cudaError_t launch(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  using C = CfgW<NR, D>;
  if (p.mode == kCluster8)
    return launch_kernel_cluster(window_tc_kernel<NR, D, true>, dim3((unsigned)p.B * p.H_kv * p.row_tiles * p.cluster),
                                 dim3(C::kThreads), C::kSmem, s, pdl, (unsigned)p.cluster, p, tmK, tmV);
  return launch_kernel(window_tc_kernel<NR, D, false>, dim3(p.shares * p.row_tiles), dim3(C::kThreads), C::kSmem, s, pdl, p, tmK, tmV);
}
template <int D>
cudaError_t launch_rows(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  if (p.rows_per_tile <= 8) return launch<8, D>(p, tmK, tmV, s, pdl);
  if (p.rows_per_tile <= 16) return launch<16, D>(p, tmK, tmV, s, pdl);
  return launch<32, D>(p, tmK, tmV, s, pdl);
}

}  // namespace

cudaError_t window_tc_prepare() {
  cudaError_t e = prepare<8, 128>();
  if (e == cudaSuccess) e = prepare<16, 128>();
  if (e == cudaSuccess) e = prepare<32, 128>();
  if (e == cudaSuccess) e = prepare<8, 64>();
  if (e == cudaSuccess) e = prepare<16, 64>();
  if (e == cudaSuccess) e = prepare<32, 64>();
  return e;
}

cudaError_t launch_window_tc(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl) {
  return p.d == 128 ? launch_rows<128>(p, tmK, tmV, s, pdl) : launch_rows<64>(p, tmK, tmV, s, pdl);
}

}  // namespace ss
