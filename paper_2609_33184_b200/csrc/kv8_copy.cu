// Rows into the 8-bit KV cache and back.
//
// A row of d values is handled by d / 16 neighbouring lanes, 16 values each: two 16-byte loads of
// bf16 and one 16-byte store of codes (write), or the reverse (read).  The row's exponent comes
// from an integer maximum over the bf16 bit patterns (a shuffle reduction over the lanes), so the
// only floating-point steps are an exact multiplication by a power of two and one rounding to
// e4m3; reading back is exact (4 significant bits times 2^e).  Memory bound: 3 d + 1 bytes per row.
#include <cuda_fp8.h>

#include "kv8.cuh"

namespace ss {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 2;   // rows in flight per thread

// Unsigned division by a launch constant: q = (mulhi(n, m) + n) >> s for n < 2^31.
struct Div {
  uint32_t d, m, s;
};
Div make_div(uint32_t d) {
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  const uint64_t m = ((1ull << 32) * ((1ull << s) - d)) / d + 1;
  return {d, (uint32_t)m, s};
}
__device__ __forceinline__ uint32_t quot(const Div& v, uint32_t n) {
  return (uint32_t)(((uint64_t)__umulhi(n, v.m) + n) >> v.s);
}

struct RowAt {
  int64_t b16;      // element offset on the bf16 side
  int64_t c8, sc;   // byte offsets of the codes and of the scale byte
  bool v, live;
  bool zero;        // (read) page outside the pool: the row reads as zeros
};

// Row number -> addresses.  Rows are numbered (request, K|V, head, row), the row fastest.
template <bool WRITE>
__device__ __forceinline__ RowAt row_at(const Copy8Params& p, const Div& dT, const Div& dH, uint32_t row, bool report) {
  RowAt a;
  uint32_t x = quot(dT, row);
  const int k = (int)(row - x * dT.d);
  const uint32_t y = quot(dH, x);
  const int h = (int)(x - y * dH.d);
  a.v = y & 1;
  const int b = (int)(y >> 1);
  const bool first = report && h == 0 && !a.v;  // one row of its kind reports
  a.live = false;
  a.zero = false;
  int n = p.cnt ? p.cnt[b] : p.T;
  if (n < 0 || n > p.T) {
    if (first && k == 0) atomicOr(p.status, WRITE ? SS_DEV_BAD_ACCEPT : SS_DEV_BAD_VALID_LEN);
    n = max(0, min(n, p.T));
  }
  if (k >= n) return a;
  int src = k;
  if (WRITE && p.idx) {
    src = p.idx[(int64_t)b * p.T + k];
    if (src < 0 || src >= p.T) {
      if (first) atomicOr(p.status, SS_DEV_BAD_ACCEPT);
      return a;
    }
  }
  const int64_t tok = (p.off ? (int64_t)p.off[b] : 0) + k;
  if (tok < 0 || tok >= p.kv.room) {
    if (first) atomicOr(p.status, WRITE ? SS_DEV_DST_OVERFLOW : SS_DEV_BAD_VALID_LEN);
    return a;
  }
  int inner, outer = outer8(p.kv, b, (int)tok, &inner);
  if (outer < 0) {
    if (first) atomicOr(p.status, SS_DEV_BAD_PAGE);
    if (WRITE) return a;
    a.zero = true;
    outer = 0;
  }
  a.live = true;
  a.b16 = b * (a.v ? p.v_sb : p.k_sb) + h * (a.v ? p.v_sh : p.k_sh) + src * (a.v ? p.v_st : p.k_st);
  a.c8 = outer * (a.v ? p.kv.v_sb : p.kv.k_sb) + h * (a.v ? p.kv.v_sh : p.kv.k_sh) + inner * (a.v ? p.kv.v_st : p.kv.k_st);
  a.sc = outer * (a.v ? p.kv.vs_sb : p.kv.ks_sb) + h * (a.v ? p.kv.vs_sh : p.kv.ks_sh) +
         inner * (a.v ? p.kv.vs_st : p.kv.ks_st);
  return a;
}

// largest finite magnitude (as bf16 bits) of two packed values and `top`
__device__ __forceinline__ uint32_t top_of(uint32_t two, uint32_t top) {
  const uint32_t lo = two & 0x7fffu, hi = (two >> 16) & 0x7fffu;
  if (lo < 0x7f80u) top = max(top, lo);
  if (hi < 0x7f80u) top = max(top, hi);
  return top;
}
__device__ __forceinline__ uint32_t codes_of(uint32_t two, float inv) {
  const float2 v = make_float2(__uint_as_float(two << 16) * inv, __uint_as_float(two & 0xffff0000u) * inv);
  return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t bf16_of(uint32_t two, float scale) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
  const __nv_bfloat162 o = __floats2bfloat162_rn(v.x * scale, v.y * scale);
  return *reinterpret_cast<const uint32_t*>(&o);
}

template <int D>
__global__ void __launch_bounds__(kThreads) write8_kernel(const __grid_constant__ Copy8Params p, const Div dT,
                                                          const Div dH, const uint32_t rows) {
  constexpr int LPR = D / 16, RPB = kThreads / LPR;
  const int part = threadIdx.x % LPR;
  const uint32_t row0 = blockIdx.x * (RPB * kUnroll) + threadIdx.x / LPR;
  RowAt at[kUnroll];
  uint4 raw[kUnroll][2];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t row = row0 + u * RPB;
    at[u].live = false;
    if (row < rows) at[u] = row_at<true>(p, dT, dH, row, part == 0);
    raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
    if (at[u].live) {
      const uint4* src = reinterpret_cast<const uint4*>((at[u].v ? p.V : p.K) + at[u].b16 + part * 16);
      raw[u][0] = __ldcs(src);
      raw[u][1] = __ldcs(src + 1);
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t w[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w,
                           raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = top_of(w[j], top);
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    // top = (1 + f / 128) 2^(E - 127) against 448 = (1 + 96 / 128) 2^8
    const int e = max(kMinExp8, min(kMaxExp8, (int)(top >> 7) - 127 - 8 + ((top & 127u) > 96u ? 1 : 0)));
    const float inv = pow2_8(-e);
    if (!at[u].live) continue;
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = codes_of(w[2 * j], inv) | (codes_of(w[2 * j + 1], inv) << 16);
    *reinterpret_cast<uint4*>((at[u].v ? p.kv.V : p.kv.K) + at[u].c8 + part * 16) = make_uint4(c[0], c[1], c[2], c[3]);
    if (part == 0) (at[u].v ? p.kv.Vs : p.kv.Ks)[at[u].sc] = (uint8_t)(e + 127);
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads) read8_kernel(const __grid_constant__ Copy8Params p, const Div dT,
                                                         const Div dH, const uint32_t rows) {
  constexpr int LPR = D / 16, RPB = kThreads / LPR;
  const int part = threadIdx.x % LPR;
  const uint32_t row0 = blockIdx.x * (RPB * kUnroll) + threadIdx.x / LPR;
  RowAt at[kUnroll];
  uint4 raw[kUnroll];
  uint32_t sc[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t row = row0 + u * RPB;
    at[u].live = false;
    if (row < rows) at[u] = row_at<false>(p, dT, dH, row, part == 0);
    raw[u] = make_uint4(0, 0, 0, 0);
    sc[u] = 127;
    if (at[u].live && !at[u].zero) {
      raw[u] = __ldcs(reinterpret_cast<const uint4*>((at[u].v ? p.kv.V : p.kv.K) + at[u].c8 + part * 16));
      sc[u] = (at[u].v ? p.kv.Vs : p.kv.Ks)[at[u].sc];
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (!at[u].live) continue;
    const float scale = scale8(sc[u]);
    const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[2 * j] = bf16_of(w[j] & 0xffffu, scale);
      o[2 * j + 1] = bf16_of(w[j] >> 16, scale);
    }
    uint4* dst = reinterpret_cast<uint4*>((at[u].v ? p.V : p.K) + at[u].b16 + part * 16);
    dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
    dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

template <bool WRITE>
cudaError_t launch_copy(const Copy8Params& p, cudaStream_t s) {
  const uint32_t rows = (uint32_t)p.B * p.T * p.H_kv * 2;  // below 2^31 (checked by the caller)
  const uint32_t per = kThreads / (p.d / 16) * kUnroll;
  const dim3 grid((rows + per - 1) / per), block(kThreads);
  const Div dT = make_div(p.T), dH = make_div(p.H_kv);
  if (p.d == 128) return launch_kernel(WRITE ? write8_kernel<128> : read8_kernel<128>, grid, block, 0, s, false, p, dT, dH, rows);
  return launch_kernel(WRITE ? write8_kernel<64> : read8_kernel<64>, grid, block, 0, s, false, p, dT, dH, rows);
}

}  // namespace

cudaError_t launch_kv8_write(const Copy8Params& p, cudaStream_t s) { return launch_copy<true>(p, s); }
cudaError_t launch_kv8_read(const Copy8Params& p, cudaStream_t s) { return launch_copy<false>(p, s); }

}  // namespace ss
