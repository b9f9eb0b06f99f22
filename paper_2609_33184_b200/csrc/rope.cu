// Rotary positions on Q and K rows, and rows that join a cache (bf16 or 8 bits), K rotated on the way.
//
// Pair i of a row at position p turns by p * f_i, which for far positions is thousands of revolutions: as an
// fp32 product (24 bits) the angle of the fastest pair is off by 2^-7 at p = 2^17.  f_i is held as revolutions
// in units of 2^-64 instead (ss_rope_init), so p * f_i is one integer product whose overflow drops the whole
// revolutions, off by at most 2^-65 * |p| <= 2^-34 revolutions; sine and cosine come from the upper 32 bits.  Values are
// turned in fp32 and rounded once, to bf16.  8 bits: the codes are those of the rounded bf16 rows, so a row is
// the same bits as rotated and then written with ss_kv8_write.
//
// A row of d values is handled by d / 16 neighbouring lanes, each 8 values from two places half of the turning
// part apart: that makes 8 pairs in either layout, and 16-byte accesses contiguous over the lanes.  A thread
// keeps the sines of its 8 pairs for the rows of one token that it handles, one after the other over the heads
// (Q, K, V).  Memory bound: 4 d bytes per row.
#include <cuda_fp8.h>

#include "rope.cuh"

namespace ss {
namespace {

constexpr int kThreads = 128;

// A block takes 2^shift consecutive tokens of a request and `heads` rows of Q, of K or of V (q_blocks and twice
// kv_blocks of them): `lanes` rows side by side, one after the other beyond.  JOINT: all rows of its tokens.
struct Plan {
  int shift, lanes, heads;
  int token_blocks, q_blocks, kv_blocks, head_blocks;
};

__device__ __forceinline__ float lo_f(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float hi_f(uint32_t two) { return __uint_as_float(two & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 o = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&o);
}

// Sine and cosine of t / 2^32 revolutions.  The nearest quarter is taken off in the integer (exact) and |x| <= pi / 4 is
// left, where the Taylor series to x^9 and x^8 are off by 2^-29 and 2^-25; x is rounded twice (2^-24 at most).  (With
// sincospif 54.0 us against 53.1 for 16,400 tokens of 40 rows; its argument, a whole revolution in fp32, was rounded more
// coarsely: of 201 million bf16 values 6,353 fell on the other side of a rounding boundary, now 4,025.)
__device__ __forceinline__ void sincos_turn(int32_t t, float* s, float* c) {
  const uint32_t quarter = ((uint32_t)t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)((uint32_t)t - (quarter << 30)) * 1.46291807926715968105e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float a = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float b = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float u = quarter & 1 ? b : a, v = quarter & 1 ? a : b;
  *s = __uint_as_float(__float_as_uint(u) ^ ((quarter & 2) << 30));
  *c = __uint_as_float(__float_as_uint(v) ^ ((quarter + 1 & 2) << 30));
}

// The sines of a thread's 8 pairs.
struct Turn {
  float c[8], s[8];
};
// (cos x - sin y, sin x + cos y)
__device__ __forceinline__ void turn2(float& x, float& y, float c, float s) {
  const float u = fmaf(x, c, -(y * s));
  y = fmaf(x, s, y * c);
  x = u;
}
// Half-split layout: value k of the first place pairs with value k of the second.  Interleaved: neighbours.
template <bool INTER>
__device__ __forceinline__ void turn_row(uint4 (&raw)[2], const Turn& t) {
  uint32_t a[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w}, b[4] = {raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float a0 = lo_f(a[k]), a1 = hi_f(a[k]), b0 = lo_f(b[k]), b1 = hi_f(b[k]);
    if (INTER) {
      turn2(a0, a1, t.c[k], t.s[k]);
      turn2(b0, b1, t.c[4 + k], t.s[4 + k]);
    } else {
      turn2(a0, b0, t.c[2 * k], t.s[2 * k]);
      turn2(a1, b1, t.c[2 * k + 1], t.s[2 * k + 1]);
    }
    a[k] = pack(a0, a1);
    b[k] = pack(b0, b1);
  }
  raw[0] = make_uint4(a[0], a[1], a[2], a[3]);
  raw[1] = make_uint4(b[0], b[1], b[2], b[3]);
}

// Largest finite magnitude (bf16 bits) of a thread's 16 values.
__device__ __forceinline__ uint32_t top_of(const uint4 (&raw)[2]) {
  const uint32_t x[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
  uint32_t two = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) two = __vmaxu2(two, x[j] & 0x7fff7fffu);
  uint32_t top = max(two & 0xffffu, two >> 16);
  if (__any_sync(0xffffffffu, top >= 0x7f80u)) {  // infinities and NaN do not count
    top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t lo = x[j] & 0x7fffu, hi = (x[j] >> 16) & 0x7fffu;
      if (lo < 0x7f80u) top = max(top, lo);
      if (hi < 0x7f80u) top = max(top, hi);
    }
  }
  return top;
}
__device__ __forceinline__ uint2 codes_of(const uint4& raw, float inv) {
  const uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t c[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    c[j] = __nv_cvt_float2_to_fp8x2(make_float2(lo_f(x[j]) * inv, hi_f(x[j]) * inv), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}

// BITS of the cache (0: rows go to Qo, Ko); U rows in flight per thread.  The compiler is held to 64, 72 or 80 registers
// (left alone it works out all sines side by side in 96 to 104: 194 us against 186 for a batch of prompts).
template <int D, int BITS, bool INTER, int U, bool JOINT>
__global__ void __launch_bounds__(kThreads, JOINT || BITS == 8 ? 8 : U == 4 ? 6 : 7) rope_kernel(const __grid_constant__ RopeParams p, const Plan plan) {
  constexpr int LPR = D / 16;
  __shared__ uint64_t freq_s[kRopePairs];
  __shared__ uint8_t axis_s[kRopePairs];
  const int tid = threadIdx.x, rot = p.rope.rot_dim;
  if (tid < rot / 2) {
    freq_s[tid] = p.rope.turn[tid];
    axis_s[tid] = p.rope.axis[tid];
  }
  __syncthreads();
  pdl_wait_prior();
  pdl_launch_dependents();
  int x = blockIdx.x;
  const int tb = x % plan.token_blocks;
  x /= plan.token_blocks;
  const int hb = x % plan.head_blocks, b = x / plan.head_blocks;
  int n = p.cnt ? p.cnt[b] : p.T;
  const bool report = tb == 0 && hb == 0;
  if (n < 0 || n > p.T) {
    if (tid == 0 && report) atomicOr(p.status, SS_DEV_BAD_ACCEPT);
    n = max(0, min(n, p.T));
  }
  const int slot = tid / LPR, part = tid % LPR, head = slot >> plan.shift;  // (of the heads side by side)
  const int k = (tb << plan.shift) + (slot & ((1 << plan.shift) - 1));       // row of the call
  if ((tb << plan.shift) >= n) return;
  const bool is_q = !JOINT && hb < plan.q_blocks, is_v = !JOINT && hb >= plan.q_blocks + plan.kv_blocks;
  const int from = (is_q ? hb : is_v ? hb - plan.q_blocks - plan.kv_blocks : hb - plan.q_blocks) * plan.heads;
  const int to = JOINT ? p.H_q + (BITS ? 2 : 1) * p.H_kv : min(from + plan.heads, is_q ? p.H_q : p.H_kv);  // the block's heads
  const int64_t off = p.off ? (int64_t)p.off[b] : 0, tok = off + k;

  // the input row
  bool live = k < n;
  int src = k;
  const bool one = part == 0 && head == 0 && hb == 0;  // who reports a row
  if (BITS && live && p.idx) {
    src = p.idx[(int64_t)b * p.T + k];
    if (src < 0 || src >= p.T) {
      if (one) atomicOr(p.status, SS_DEV_BAD_ACCEPT);
      live = false;
      src = 0;
    }
  }

  // this thread's two places in a row
  const bool turning = part * 16 < rot;
  const int at0 = turning ? part * 8 : rot + (part - rot / 16) * 8;
  const int at1 = turning ? rot / 2 + part * 8 : rot + (D - rot) / 2 + (part - rot / 16) * 8;
  // U rows on their way, the first ones before the token's place is looked up and the sines are worked out (16,400 tokens
  // of 40 rows, three axes: 54.8 -> 53.1 us)
  const int64_t in_sh = is_q ? p.q_sh : is_v ? p.v_sh : p.k_sh, step = plan.lanes * in_sh;
  const uint16_t* at = (is_q   ? p.Q + b * p.q_sb + src * p.q_st
                        : is_v ? p.V + b * p.v_sb + src * p.v_st
                               : p.K + b * p.k_sb + src * p.k_st) + (from + head) * in_sh;
  uint4 raw[U][2];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
      if (JOINT) {
        const int h = h0 + u, k = h - p.H_q, v = k - p.H_kv;
        at = h < p.H_q ? p.Q + b * p.q_sb + src * p.q_st + h * p.q_sh
             : v < 0   ? p.K + b * p.k_sb + src * p.k_st + k * p.k_sh
                       : p.V + b * p.v_sb + src * p.v_st + v * p.v_sh;
      }
      if (live && h0 + u * plan.lanes < to) {
        raw[u][0] = __ldcs(reinterpret_cast<const uint4*>(at + at0));
        raw[u][1] = __ldcs(reinterpret_cast<const uint4*>(at + at1));
      }
      if (!JOINT) at += step;
    }
  };
  load(JOINT ? 0 : from + head);

  // (cache) the token's place
  bool store = live;
  uint64_t outer = (uint64_t)b, inner = (uint64_t)tok;
  if (BITS && live) {
    if (tok < 0 || tok >= p.kv.room) {
      if (one) atomicOr(p.status, SS_DEV_DST_OVERFLOW);
      store = false;
    }
    if (store && p.kv.page_table) {
      const uint32_t t = (uint32_t)tok, pg = p.kv.page_log2 >= 0 ? t >> p.kv.page_log2 : t / (uint32_t)p.kv.page_size;
      inner = t - pg * p.kv.page_size;
      const uint32_t id = (uint32_t)p.kv.page_table[(int64_t)b * p.kv.pages_per_req + pg];
      if (id >= (uint32_t)p.kv.n_outer) {
        if (one) atomicOr(p.status, SS_DEV_BAD_PAGE);
        store = false;
      }
      outer = id;
    }
  }

  // the sines of this thread's pairs
  Turn t;
  if (turning && live && !is_v) {
    int64_t pos[kRopeAxes];
#pragma unroll
    for (int a = 0; a < kRopeAxes; ++a)
      pos[a] = p.pos && a < p.rope.n_axes ? (int64_t)p.pos[((int64_t)a * p.B + b) * p.T + src] : tok;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int pair = INTER ? (j < 4 ? part * 4 + j : rot / 4 + part * 4 + j - 4) : part * 8 + j;
      const int a = axis_s[pair];
      const int64_t at = a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : pos[3];
      const uint64_t turns = freq_s[pair] * (uint64_t)at;                // whole revolutions overflow
      sincos_turn((int32_t)(turns >> 32), &t.s[j], &t.c[j]);
      t.s[j] *= p.rope.magnitude;
      t.c[j] *= p.rope.magnitude;
    }
  }

  // The block's rows: put(head, row) stores one.  As often for every lane of a warp.
  auto rows = [&](bool turn, bool ok, auto put) {
#pragma unroll 1
    for (int h0 = from + head;;) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (turn) turn_row<INTER>(raw[u], t);
        put(h0 + u * plan.lanes, ok && h0 + u * plan.lanes < to, raw[u]);
      }
      h0 += U * plan.lanes;
      if (h0 - head >= to) break;
      load(h0);
    }
  };
  auto to_rows = [&](uint16_t* out, int64_t out_sh) {
    return [=](int h, bool ok, const uint4 (&raw)[2]) {
      if (!ok) return;
      uint16_t* row = out + h * out_sh;
      *reinterpret_cast<uint4*>(row + at0) = raw[0];
      *reinterpret_cast<uint4*>(row + at1) = raw[1];
    };
  };
  auto to_cache = [&](uint8_t* out, int64_t out_sh, uint8_t* scale, int64_t scale_sh) {
    return [=](int h, bool ok, const uint4 (&raw)[2]) {
      uint8_t* row = out + h * out_sh;
      if (BITS == 16) {
        if (!ok) return;
        __stcs(reinterpret_cast<uint4*>(row + 2 * at0), raw[0]);
        __stcs(reinterpret_cast<uint4*>(row + 2 * at1), raw[1]);
      } else {
        uint32_t top = top_of(raw);  // (by all lanes: a row's are neighbours)
#pragma unroll
        for (int o = LPR / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (!ok) return;
        // top = (1 + f / 128) 2^(E - 127) against 448 = (1 + 96 / 128) 2^8
        const int e = max(kMinExp8, min(kMaxExp8, (int)((top + 31u) >> 7) - 127 - 8));
        const float inv = pow2_8(-e);
        __stcs(reinterpret_cast<uint2*>(row + at0), codes_of(raw[0], inv));
        __stcs(reinterpret_cast<uint2*>(row + at1), codes_of(raw[1], inv));
        if (part == 0) scale[h * scale_sh] = (uint8_t)(e + 127);
      }
    };
  };
  if (JOINT) {
    const auto put_q = to_rows(p.Qo + b * p.qo_sb + src * p.qo_st, p.qo_sh);
    const auto put_k = to_rows(p.Ko + b * p.ko_sb + src * p.ko_st, p.ko_sh);
    const auto put_k8 = to_cache(p.kv.K + outer * p.kv.k_sb + inner * p.kv.k_st, p.kv.k_sh,
                                 p.kv.Ks + outer * p.kv.ks_sb + inner * p.kv.ks_st, p.kv.ks_sh);
    const auto put_v8 = to_cache(p.kv.V + outer * p.kv.v_sb + inner * p.kv.v_st, p.kv.v_sh,
                                 p.kv.Vs + outer * p.kv.vs_sb + inner * p.kv.vs_st, p.kv.vs_sh);
#pragma unroll 1
    for (int h0 = 0;;) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u, k = h - p.H_q, v = k - p.H_kv;
        if (h >= to) break;
        if (v < 0 && turning) turn_row<INTER>(raw[u], t);
        if (k < 0) put_q(h, live, raw[u]);
        else if (BITS == 0) put_k(k, live, raw[u]);
        else if (v < 0) put_k8(k, store, raw[u]);
        else put_v8(v, store, raw[u]);
      }
      h0 += U;
      if (h0 >= to) break;
      load(h0);
    }
  } else if (is_q) {
    rows(turning, live, to_rows(p.Qo + b * p.qo_sb + src * p.qo_st, p.qo_sh));
  } else if (BITS == 0) {
    rows(turning, live, to_rows(p.Ko + b * p.ko_sb + src * p.ko_st, p.ko_sh));
  } else if (!is_v) {
    rows(turning, store, to_cache(p.kv.K + outer * p.kv.k_sb + inner * p.kv.k_st, p.kv.k_sh,
                           p.kv.Ks + outer * p.kv.ks_sb + inner * p.kv.ks_st, p.kv.ks_sh));
  } else {
    rows(false, store, to_cache(p.kv.V + outer * p.kv.v_sb + inner * p.kv.v_st, p.kv.v_sh,
                         p.kv.Vs + outer * p.kv.vs_sb + inner * p.kv.vs_st, p.kv.vs_sh));
  }
}

template <int D, int BITS, bool INTER, int U, bool JOINT = false>
cudaError_t launch_rows(const RopeParams& p, int heads, cudaStream_t s, bool pdl) {
  constexpr int kSlots = kThreads * 16 / D;
  Plan plan = {};
  while (1 << plan.shift < p.T && 1 << plan.shift < kSlots) ++plan.shift;
  plan.lanes = kSlots >> plan.shift;
  plan.heads = heads * plan.lanes;
  plan.token_blocks = (p.T + (1 << plan.shift) - 1) >> plan.shift;
  plan.q_blocks = (p.H_q + plan.heads - 1) / plan.heads;
  plan.kv_blocks = (p.H_kv + plan.heads - 1) / plan.heads;
  plan.head_blocks = JOINT ? 1 : plan.q_blocks + (BITS ? 2 : 1) * plan.kv_blocks;
  const dim3 grid((unsigned)plan.token_blocks * plan.head_blocks * p.B);  // below 2^31: see the caller
  return launch_kernel(rope_kernel<D, BITS, INTER, U, JOINT>, grid, dim3(kThreads), 0, s, pdl, p, plan);
}
template <int D, int BITS, bool INTER>
cudaError_t launch_layout(const RopeParams& p, cudaStream_t s, bool pdl) {
  const int all = p.H_q + p.H_kv + (BITS ? p.H_kv : 0);
  // large: more rows than 8 blocks per SM would take, a row a thread.  There a thread turns 8 rows with its sines, 4 in
  // flight (2 into 8 bits, whose conversions want the registers: 66 -> 59 us for 49,000 tokens of 8 heads); 4 rows
  // instead of 8: 207 us against 187 for a batch of prompts, 16: 188, and 6.2 against 4.7 for 1024 tokens.  Small
  // calls take two rows a thread (one: 4.9 us against 2.9 for 256 tokens of 48 rows, as much for less).
  const bool large = (int64_t)p.B * p.T * all > (int64_t)8 * kNumSM * kThreads * 16 / D;
  constexpr int kU = BITS == 8 ? 2 : 4;
  // Few heads (a GPU's part of a model's): a token's rows in one block, or its sines and its start would be paid for two or
  // three blocks (6 x 9000 tokens, 2 + 1 heads, rows into bf16 38.4 -> 22.2 us, 4 + 1 41.5 -> 30.1, 6 + 1 48.0 -> 38.3, K and V
  // of 4 35.3 and 37.2; into 8 bits 2 + 1 33.9 -> 24.2, 4 + 1 37.7 -> 31.9, 8 + 1 47.1 and 49.6, K and V of 4 35.5 and 38.9).
  const int few = BITS == 8 || !p.H_q ? 6 : 8;
  if (large && all <= few && p.T >= kThreads * 16 / D) return launch_rows<D, BITS, INTER, 2, true>(p, all, s, pdl);
  return large ? launch_rows<D, BITS, INTER, kU>(p, 8, s, pdl) : launch_rows<D, BITS, INTER, 2>(p, 2, s, pdl);
}
template <int D, int BITS>
cudaError_t launch_bits(const RopeParams& p, cudaStream_t s, bool pdl) {
  return p.rope.interleaved ? launch_layout<D, BITS, true>(p, s, pdl) : launch_layout<D, BITS, false>(p, s, pdl);
}
template <int D>
cudaError_t launch_dim(const RopeParams& p, cudaStream_t s, bool pdl) {
  return p.bits == 16 ? launch_bits<D, 16>(p, s, pdl) : p.bits == 8 ? launch_bits<D, 8>(p, s, pdl) : launch_bits<D, 0>(p, s, pdl);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, cudaStream_t s, bool pdl) {
  return p.d == 128 ? launch_dim<128>(p, s, pdl) : launch_dim<64>(p, s, pdl);
}

}  // namespace ss
