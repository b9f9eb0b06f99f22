// Attention over the 8-bit KV cache, and over a window of it or of a bf16 one, on the CUDA cores: any page
// size, any strides the tensor maps cannot express, and head dims 64 and 128.
//
// A CTA walks its share of the tiles (kv8.cuh) for tiles of 8 query rows.  Each of its four warps
// takes 32 keys of a 128-token tile, one per lane: the lane reads its key's codes 16 bytes at a
// time and forms the 8 scores in fp32 against Q in shared memory (the key's scale 2^e multiplies
// the finished sum, exactly); running maximum and sum per warp and row, in fp32; weights times the
// value scale go through shared memory and every lane accumulates d / 32 head dims over the 32
// keys.  The warps' states meet when a segment ends.  Bound by conversions and shared-memory
// reads, not by memory: it is the general form, not the fast one (decoding, 16 x 32768 tokens, 8 heads of 128, 4 rows:
// 2600 us for pages of 4, 24 or 192 tokens, the tensor cores take 166 for pages of 64; 32 rows 10500 against 184).
#include <cuda_fp8.h>

#include "kv8.cuh"

namespace ss {
namespace {

constexpr int kRT = kMinRows8;

__device__ __forceinline__ float2 f2_of_e4m3x2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float warp_max8(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum8(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// 16 values of a row of the cache, from value c on (zeros where there is no row).
template <int BITS>
__device__ __forceinline__ void load16(const uint8_t* row, int c, bool there, float2 (&x)[8]) {
  if (BITS == 8) {
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (there) raw = *reinterpret_cast<const uint4*>(row + c);
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = f2_of_e4m3x2((w[j / 2] >> (16 * (j & 1))) & 0xffffu);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (there) raw = *reinterpret_cast<const uint4*>(row + 2 * c + 16 * h);
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[4 * h + j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    }
  }
}
template <int BITS>
__device__ __forceinline__ float2 load2(const uint8_t* row, int c) {
  if (BITS == 8) return f2_of_e4m3x2(*reinterpret_cast<const uint16_t*>(row + c));
  const uint32_t w = *reinterpret_cast<const uint32_t*>(row + 2 * c);
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <int D, int BITS, bool WIN>
__global__ void __launch_bounds__(128) attn8_simt_kernel(const __grid_constant__ Attn8Params p) {
  constexpr int CPL = D / 32;  // head dims per lane in the output
  __shared__ __align__(16) float q_s[kRT][D];
  __shared__ __align__(16) float w_s[4][32][kRT];
  __shared__ float2 ml_s[4][kRT];
  __shared__ float a_s[4][kRT][D];
  __shared__ int pos_s[kRT];   // (window) the rows' positions
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait_prior();
  pdl_launch_dependents();
  const Share8 share = find_share8<WIN>(p);
  Seg8 g;
  for (bool more = seg_first8<WIN>(p, share, &g); more; more = seg_next8<WIN>(p, share, &g)) {
    __syncthreads();  // the previous segment's shared memory has been read
    Win8 w = {};
    if (WIN) {
      w = win8(p, g.b);
      if (tid < g.nrows) pos_s[tid] = w.first + depth8(p, g.b, (g.row0 + tid) % p.T_q);
    }
    for (int i = tid; i < kRT * D; i += 128) {
      const int r = i / D, c = i % D;
      float v = 0.f;
      if (r < g.nrows) {
        const int rg = g.row0 + r, h = g.kvh * p.G + rg / p.T_q, t = rg % p.T_q;
        v = __bfloat162float(p.Q[g.b * p.q_sb + h * p.q_sh + t * p.q_st + c]);
        // (an infinite query too makes its scores NaN, whatever the signs of its products)
        if (!(fabsf(v) < INFINITY)) v = __int_as_float(0x7fffffff);
      }
      q_s[r][c] = v;
    }
    __syncthreads();
    float m[kRT], l[kRT], acc[kRT][CPL];
#pragma unroll
    for (int r = 0; r < kRT; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) acc[r][c] = 0.f;
    }
    for (int t = g.t0; t < g.t1; ++t) {
      const int tok0 = t * kTok8 + warp * 32, v_tok = tok0 + lane;
      if (tok0 >= g.len) continue;
      const bool ok = v_tok < g.len;
      const int tok = WIN ? win_token8(w, v_tok) : v_tok;
      const uint32_t reach = WIN ? win_reach8(p, w, tok) : 0u;
      int inner = 0, outer = -1;
      if (ok) {
        outer = outer8(p.kv, g.b, tok, &inner);
        if (outer < 0) atomicOr(p.status, SS_DEV_BAD_PAGE);  // reads as zeros
      }
      float s[kRT], vs = 0.f;
#pragma unroll
      for (int r = 0; r < kRT; ++r) s[r] = 0.f;
      if (ok) {  // (a page outside the pool is zeros: 0 * q, NaN where the query is)
        const uint8_t* k = p.kv.K + outer * p.kv.k_sb + g.kvh * p.kv.k_sh + inner * p.kv.k_st;
#pragma unroll 2
        for (int c16 = 0; c16 < D; c16 += 16) {
          float2 x[8];
          load16<BITS>(k, c16, outer >= 0, x);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 k01 = x[2 * j], k23 = x[2 * j + 1];
#pragma unroll
            for (int r = 0; r < kRT; ++r) {
              const float4 q = *reinterpret_cast<const float4*>(&q_s[r][c16 + j * 4]);
              s[r] = fmaf(q.x, k01.x, fmaf(q.y, k01.y, fmaf(q.z, k23.x, fmaf(q.w, k23.y, s[r]))));
            }
          }
        }
        uint32_t ek = 127, ev = 127;
        if (BITS == 8 && outer >= 0) {
          ek = p.kv.Ks[outer * p.kv.ks_sb + g.kvh * p.kv.ks_sh + inner * p.kv.ks_st];
          ev = p.kv.Vs[outer * p.kv.vs_sb + g.kvh * p.kv.vs_sh + inner * p.kv.vs_st];
        }
        const float ks = scale8(byte8(ek)) * p.scale_log2;
        vs = scale8(byte8(ev));
#pragma unroll
        for (int r = 0; r < kRT; ++r) s[r] *= ks;
      }
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
        const bool seen = ok && (!WIN || (r < g.nrows && win_sees8(pos_s[r], tok, reach)));
        const float x = seen ? s[r] : -INFINITY;
        const float top = fmaxf(m[r], warp_max8(x));
        const float f = (m[r] == top) ? 1.f : exp2f(m[r] - top);  // (equal also when both are -inf)
        // (no finite score so far: weight 0, except that a NaN score has to show)
        const float w = !seen ? 0.f : (top == -INFINITY && x == x) ? 0.f : exp2f(x - top);
        m[r] = top;
        l[r] = fmaf(l[r], f, w);
#pragma unroll
        for (int c = 0; c < CPL; ++c) acc[r][c] *= f;
        w_s[warp][lane][r] = w * vs;
      }
      __syncwarp();
      const int n = min(32, g.len - tok0);
#pragma unroll 4
      for (int j = 0; j < n; ++j) {
        const int o = __shfl_sync(0xffffffffu, outer, j), in = __shfl_sync(0xffffffffu, inner, j);
        if (o < 0) continue;
        const uint8_t* v = p.kv.V + o * p.kv.v_sb + g.kvh * p.kv.v_sh + in * p.kv.v_st + lane * CPL * (BITS / 8);
        float x[CPL];
#pragma unroll
        for (int c = 0; c < CPL; c += 2) {
          const float2 a = load2<BITS>(v, c);
          x[c] = a.x;
          x[c + 1] = a.y;
        }
        float wr[kRT];
        *reinterpret_cast<float4*>(wr) = *reinterpret_cast<const float4*>(&w_s[warp][j][0]);
        *reinterpret_cast<float4*>(wr + 4) = *reinterpret_cast<const float4*>(&w_s[warp][j][4]);
#pragma unroll
        for (int r = 0; r < kRT; ++r)
#pragma unroll
          for (int c = 0; c < CPL; ++c) acc[r][c] = fmaf(wr[r], x[c], acc[r][c]);
      }
      __syncwarp();
    }
    // the four warps' states
#pragma unroll
    for (int r = 0; r < kRT; ++r) {
      const float lr = warp_sum8(l[r]);
      if (lane == 0) ml_s[warp][r] = make_float2(m[r], lr);
#pragma unroll
      for (int c = 0; c < CPL; ++c) a_s[warp][r][lane * CPL + c] = acc[r][c];
    }
    __syncthreads();
    const bool whole = g.t0 == 0 && g.t1 == g.n;
    float* slot = whole ? nullptr : slot8(p, share, g.start, share.idx);
    for (int r = tid / D; r < g.nrows; r += 128 / D) {
      const int c = tid % D;
      float M = -INFINITY, L = 0.f, A = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        if (ml_s[w][r].y != 0.f) M = fmaxf(M, ml_s[w][r].x);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (ml_s[w][r].y == 0.f) continue;
        const float f = ml_s[w][r].x == M ? 1.f : exp2f(ml_s[w][r].x - M);
        L = fmaf(f, ml_s[w][r].y, L);
        A = fmaf(f, a_s[w][r][c], A);
      }
      if (whole) {
        if (c == 0) put_ml8(p, g, r, M, L);
        put_a8(p, g, r, c, L, A);
      } else {
        if (c == 0) reinterpret_cast<float2*>(slot)[r] = make_float2(M, L);
        if (c == 0 && g.t0 == 0 && !p.O) put_cut8(p, share, g, r);
        slot[4 * p.rows_per_tile + r * D + c] = A;
      }
    }
  }
  if ((int)blockIdx.x < p.B) put_empty8<WIN>(p, tid, 128);
  if (WIN && p.depth && warp == 0) check_depths8(p);
}

}  // namespace

cudaError_t launch_attn8_simt(const Attn8Params& p, int bits, cudaStream_t s, bool pdl) {
  const dim3 grid(p.shares * p.row_tiles), block(128);
  auto kernel = !p.window   ? (p.d == 128 ? attn8_simt_kernel<128, 8, false> : attn8_simt_kernel<64, 8, false>)
                : bits == 8 ? (p.d == 128 ? attn8_simt_kernel<128, 8, true> : attn8_simt_kernel<64, 8, true>)
                            : (p.d == 128 ? attn8_simt_kernel<128, 16, true> : attn8_simt_kernel<64, 16, true>);
  return launch_kernel(kernel, grid, block, 0, s, pdl, p);
}

}  // namespace ss
