// Rows into the 8-bit KV cache and back.
//
// A row of d values is handled by d / 16 neighbouring lanes, twice 8 values each, half a row apart: 16-byte
// accesses of bf16 and 8-byte accesses of codes, each contiguous over the lanes (32 contiguous bytes a
// lane would leave every access with half of each sector).  The row's exponent comes
// from an integer maximum over the bf16 bit patterns (a shuffle reduction over the lanes), so the
// only floating-point steps are an exact multiplication by a power of two and one rounding to
// e4m3; reading back is exact (4 significant bits times 2^e).  Memory bound: 3 d + 1 bytes per row.
#include <cuda_fp8.h>

#include "kv8.cuh"

namespace ss {
namespace {

constexpr int kThreads = 128;

// U rows in flight per thread: 4 for calls that fill the GPU, 1 for small ones, which want short
// threads and many blocks (102,000 prompt tokens of 8 heads, blocks of 256: 110 us with 4, 118 with 2, 158
// with 1; 32 requests' accepted tokens: 4.4, 2.8 and 2.4 us).  Blocks of 128 threads: 99 us against 107 with
// 256.  Stores go past L2's other contents (__stcs): 157 us against 191 for 165,000 tokens read back.  Both
// large cases then run at the copy rate.
//
// A block takes U * kThreads / (d / 16) rows: 2^shift consecutive tokens (T of them for short calls) of
// as many (K|V, head) pairs of one request as that makes, so the request, its count and its offset are
// the block's and a row's place costs shifts.  (Rows numbered through and divided down took 183 us for
// 102,000 prompt tokens of 8 heads instead of the time below.)
struct Plan {
  int shift;                   // log2 of the tokens of a block
  int pairs;                   // pairs of a block
  int token_blocks, pair_blocks;
};

struct Block {
  int b, k0, pair0, n;   // request, first row, first pair, rows that the call covers
  int64_t off;
};
template <bool WRITE>
__device__ __forceinline__ Block block_at(const Copy8Params& p, const Plan& plan) {
  Block w;
  int x = blockIdx.x;
  const int tb = x % plan.token_blocks;
  x /= plan.token_blocks;
  const int pb = x % plan.pair_blocks;
  w.b = x / plan.pair_blocks;
  w.k0 = tb << plan.shift;
  w.pair0 = pb * plan.pairs;
  w.n = p.cnt ? p.cnt[w.b] : p.T;
  w.off = p.off ? (int64_t)p.off[w.b] : 0;
  if (w.n < 0 || w.n > p.T) {
    if (threadIdx.x == 0 && tb == 0 && pb == 0) atomicOr(p.status, WRITE ? SS_DEV_BAD_ACCEPT : SS_DEV_BAD_VALID_LEN);
    w.n = max(0, min(w.n, p.T));
  }
  return w;
}

// One (K|V, head) pair of a request: where its rows are on both sides.
struct Pair {
  uint16_t* rows;        // bf16 row 0
  uint8_t *codes, *scales;   // outer index 0, token 0
  uint64_t row_st, code_sb, code_st, scale_sb, scale_st;
};
__device__ __forceinline__ Pair pair_at(const Copy8Params& p, int b, int pair) {
  const bool v = pair >= p.H_kv;
  const int h = v ? pair - p.H_kv : pair;
  Pair a;
  a.rows = v ? p.V + b * p.v_sb + h * p.v_sh : p.K + b * p.k_sb + h * p.k_sh;
  a.codes = v ? p.kv.V + h * p.kv.v_sh : p.kv.K + h * p.kv.k_sh;
  a.scales = v ? p.kv.Vs + h * p.kv.vs_sh : p.kv.Ks + h * p.kv.ks_sh;
  a.row_st = v ? p.v_st : p.k_st;
  a.code_sb = v ? p.kv.v_sb : p.kv.k_sb;
  a.code_st = v ? p.kv.v_st : p.kv.k_st;
  a.scale_sb = v ? p.kv.vs_sb : p.kv.ks_sb;
  a.scale_st = v ? p.kv.vs_st : p.kv.ks_st;
  return a;
}

// Row k of the call: its row on the bf16 side (src) and its place in the cache.
struct Place {
  uint32_t src, outer, inner;
  bool live, zero;       // zero: (read) in a page outside the pool, reads as zeros
};
template <bool WRITE>
__device__ __forceinline__ Place place_of(const Copy8Params& p, const Block& w, int k, bool report) {
  Place a = {(uint32_t)k, 0, 0, false, false};
  if (k >= w.n) return a;
  if (WRITE && p.idx) {
    const int src = p.idx[(int64_t)w.b * p.T + k];
    if (src < 0 || src >= p.T) {
      if (report) atomicOr(p.status, SS_DEV_BAD_ACCEPT);
      return a;
    }
    a.src = src;
  }
  const int64_t tok = w.off + k;
  if (tok < 0 || tok >= p.kv.room) {
    if (report) atomicOr(p.status, WRITE ? SS_DEV_DST_OVERFLOW : SS_DEV_BAD_VALID_LEN);
    return a;
  }
  a.live = true;
  a.outer = w.b;
  a.inner = (uint32_t)tok;
  if (p.kv.page_table) {
    const uint32_t t = (uint32_t)tok, pg = p.kv.page_log2 >= 0 ? t >> p.kv.page_log2 : t / (uint32_t)p.kv.page_size;
    a.inner = t - pg * p.kv.page_size;
    a.outer = (uint32_t)p.kv.page_table[(int64_t)w.b * p.kv.pages_per_req + pg];
    if (a.outer >= (uint32_t)p.kv.n_outer) {
      if (report) atomicOr(p.status, SS_DEV_BAD_PAGE);
      a.live = !WRITE;
      a.zero = true;
      a.outer = 0;
    }
  }
  return a;
}

// largest finite magnitude (as bf16 bits) of two packed values and `top`
__device__ __forceinline__ uint32_t top_of(uint32_t two, uint32_t top) {
  const uint32_t lo = two & 0x7fffu, hi = (two >> 16) & 0x7fffu;
  if (lo < 0x7f80u) top = max(top, lo);
  if (hi < 0x7f80u) top = max(top, hi);
  return top;
}
__device__ __forceinline__ uint32_t codes_of(uint32_t two, float2 inv) {
  const float2 v = __fmul2_rn(make_float2(__uint_as_float(two << 16), __uint_as_float(two & 0xffff0000u)), inv);
  return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t bf16_of(uint32_t two, float2 scale) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  const float2 v = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2*>(&h)), scale);
  const __nv_bfloat162 o = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&o);
}

// ONE: all rows of the block belong to one pair (calls of many rows), whose addresses are the block's.
template <int D, bool ONE, int U>
__global__ void __launch_bounds__(kThreads) write8_kernel(const __grid_constant__ Copy8Params p, const Plan plan) {
  constexpr int LPR = D / 16, RPB = kThreads / LPR;
  const int part = threadIdx.x % LPR;
  pdl_wait_prior();
  pdl_launch_dependents();
  const Block w = block_at<true>(p, plan);
  if (w.k0 >= w.n) return;
  Pair one;
  if (ONE) one = pair_at(p, w.b, w.pair0);
  Place at[U];
  uint4 raw[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x / LPR + u * RPB;
    const int pair = ONE ? w.pair0 : w.pair0 + (i >> plan.shift), k = w.k0 + (ONE ? i : i & ((1 << plan.shift) - 1));
    at[u] = place_of<true>(p, w, pair < 2 * p.H_kv ? k : w.n, part == 0 && pair == 0);
    raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
    if (at[u].live) {
      const Pair a = ONE ? one : pair_at(p, w.b, pair);
      const uint4* src = reinterpret_cast<const uint4*>(a.rows + at[u].src * a.row_st) + part;
      raw[u][0] = __ldcs(src);
      raw[u][1] = __ldcs(src + LPR);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t x[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w,
                           raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
    uint32_t top2 = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top2 = __vmaxu2(top2, x[j] & 0x7fff7fffu);
    uint32_t top = max(top2 & 0xffffu, top2 >> 16);
    if (__any_sync(0xffffffffu, top >= 0x7f80u)) {  // infinities and NaN do not count
      top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = top_of(x[j], top);
    }
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    // top = (1 + f / 128) 2^(E - 127) against 448 = (1 + 96 / 128) 2^8
    const int e = max(kMinExp8, min(kMaxExp8, (int)((top + 31u) >> 7) - 127 - 8));
    const float2 inv = make_float2(pow2_8(-e), pow2_8(-e));
    if (!at[u].live) continue;
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = codes_of(x[2 * j], inv) | (codes_of(x[2 * j + 1], inv) << 16);
    const int pair = ONE ? w.pair0 : w.pair0 + ((threadIdx.x / LPR + u * RPB) >> plan.shift);
    const Pair a = ONE ? one : pair_at(p, w.b, pair);
    uint2* dst = reinterpret_cast<uint2*>(a.codes + at[u].outer * a.code_sb + at[u].inner * a.code_st) + part;
    __stcs(dst, make_uint2(c[0], c[1]));
    __stcs(dst + LPR, make_uint2(c[2], c[3]));
    if (part == 0) a.scales[at[u].outer * a.scale_sb + at[u].inner * a.scale_st] = (uint8_t)(e + 127);
  }
}

template <int D, bool ONE, int U>
__global__ void __launch_bounds__(kThreads) read8_kernel(const __grid_constant__ Copy8Params p, const Plan plan) {
  constexpr int LPR = D / 16, RPB = kThreads / LPR;
  const int part = threadIdx.x % LPR;
  pdl_wait_prior();
  pdl_launch_dependents();
  const Block w = block_at<false>(p, plan);
  if (w.k0 >= w.n) return;
  Pair one;
  if (ONE) one = pair_at(p, w.b, w.pair0);
  uint16_t* to[U];
  uint2 raw[U][2];
  uint32_t sc[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x / LPR + u * RPB;
    const int pair = ONE ? w.pair0 : w.pair0 + (i >> plan.shift), k = w.k0 + (ONE ? i : i & ((1 << plan.shift) - 1));
    const Place at = place_of<false>(p, w, pair < 2 * p.H_kv ? k : w.n, part == 0 && pair == 0);
    to[u] = nullptr;
    raw[u][0] = raw[u][1] = make_uint2(0, 0);
    sc[u] = 127;
    if (at.live) {
      const Pair a = ONE ? one : pair_at(p, w.b, pair);
      to[u] = a.rows + at.src * a.row_st;
      if (!at.zero) {
        const uint2* src = reinterpret_cast<const uint2*>(a.codes + at.outer * a.code_sb + at.inner * a.code_st) + part;
        raw[u][0] = __ldcs(src);
        raw[u][1] = __ldcs(src + LPR);
        sc[u] = a.scales[at.outer * a.scale_sb + at.inner * a.scale_st];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!to[u]) continue;
    const float one_scale = scale8(byte8(sc[u]));
    const float2 scale = make_float2(one_scale, one_scale);
    const uint32_t x[4] = {raw[u][0].x, raw[u][0].y, raw[u][1].x, raw[u][1].y};
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[2 * j] = bf16_of(x[j] & 0xffffu, scale);
      o[2 * j + 1] = bf16_of(x[j] >> 16, scale);
    }
    uint4* dst = reinterpret_cast<uint4*>(to[u]) + part;
    __stcs(dst, make_uint4(o[0], o[1], o[2], o[3]));
    __stcs(dst + LPR, make_uint4(o[4], o[5], o[6], o[7]));
  }
}

template <bool WRITE, int D, int U>
cudaError_t launch_rows8(const Copy8Params& p, cudaStream_t s, bool pdl) {
  constexpr int kRows = U * kThreads * 16 / D;
  Plan plan = {0, 0, 0, 0};
  while (1 << plan.shift < p.T && 1 << plan.shift < kRows) ++plan.shift;
  plan.pairs = kRows >> plan.shift;
  plan.token_blocks = (p.T + (1 << plan.shift) - 1) >> plan.shift;
  plan.pair_blocks = (2 * p.H_kv + plan.pairs - 1) / plan.pairs;
  const dim3 grid((unsigned)plan.token_blocks * plan.pair_blocks * p.B), block(kThreads);  // below 2^31: see the caller
  auto kernel = plan.pairs == 1 ? (WRITE ? write8_kernel<D, true, U> : read8_kernel<D, true, U>)
                                : (WRITE ? write8_kernel<D, false, U> : read8_kernel<D, false, U>);
  return launch_kernel(kernel, grid, block, 0, s, pdl, p, plan);
}
template <bool WRITE>
cudaError_t launch_copy(const Copy8Params& p, cudaStream_t s, bool pdl) {
  // large: more rows than one block per SM would take with four in flight per thread
  const bool large = (int64_t)p.B * p.T * p.H_kv * 2 > (int64_t)kNumSM * 4 * kThreads * 16 / p.d;
  if (p.d == 128) return large ? launch_rows8<WRITE, 128, 4>(p, s, pdl) : launch_rows8<WRITE, 128, 1>(p, s, pdl);
  return large ? launch_rows8<WRITE, 64, 4>(p, s, pdl) : launch_rows8<WRITE, 64, 1>(p, s, pdl);
}

}  // namespace

cudaError_t launch_kv8_write(const Copy8Params& p, cudaStream_t s, bool pdl) { return launch_copy<true>(p, s, pdl); }
cudaError_t launch_kv8_read(const Copy8Params& p, cudaStream_t s, bool pdl) { return launch_copy<false>(p, s, pdl); }

}  // namespace ss
