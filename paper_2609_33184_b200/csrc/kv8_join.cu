// Joins the partial states of units that the attention launch cut (kv8.cuh): a warp per query row, so
// that many states of many rows are read by the whole GPU.  (Joined by the last CTA of each unit instead, with
// a ticket: one launch less and slower everywhere, 9.8 against 7.9 us for one request of 1024 tokens, 52
// against 48 for 131071, 55 against 29 for a round of 2 x 6909 tokens and 40 rows per kv-head.)
//
// The warp works the shares out again from the lengths.  It does so before it waits for the attention
// kernel: that kernel let this one start only after everything in front of it, the lengths' producer too,
// was complete.  Bound by two dependent reads of L2.
#include "kv8.cuh"

namespace ss {
namespace {

constexpr int kWarps = 4;
constexpr int kFlight = 16;  // states in flight

template <int D>
__global__ void __launch_bounds__(kWarps * 32) attn8_join_kernel(const __grid_constant__ Attn8Params p) {
  constexpr int CPL = D / 32;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);  // (request, kv-head, row)
  if (row >= (int64_t)p.B * p.H_kv * p.R) return;  // (the block's first warp has a row)
  Seg8 g;
  const int pair = (int)(row / p.R), rr = (int)(row - (int64_t)pair * p.R);
  g.b = pair / p.H_kv;
  g.kvh = pair - g.b * p.H_kv;
  const int rt = rr / p.rows_per_tile, r = rr - rt * p.rows_per_tile;
  g.row0 = rt * p.rows_per_tile;
  g.nrows = min(p.rows_per_tile, p.R - g.row0);
  g.n = tiles8(len8(p, g.b));
  const uint32_t units = (uint32_t)(p.H_kv * p.row_tiles);
  uint32_t sum = 0, before = 0;  // tiles of all requests, of those before g.b
  for (int b = lane; b < p.B; b += 32) {
    const uint32_t n = units * tiles8(len8(p, b));
    sum += n;
    if (b < g.b) before += n;
  }
  Share8 s = {};
  s.total = __reduce_add_sync(0xffffffffu, sum);
  before = __reduce_add_sync(0xffffffffu, before);
  int i0 = 0, n = 0;
  const float *first = nullptr, *rest = nullptr;
  if (g.n > 0) {
    set_shares8(p, kCtas8, &s);
    g.start = before + (uint32_t)(g.kvh * p.row_tiles + rt) * g.n;
    i0 = min((int)share_of8(s, g.start), kCtas8 - 1);  // (no address depends on more than these two)
    n = min((int)share_of8(s, g.start + g.n - 1), kCtas8 - 1) - i0 + 1;
    first = slot8(p, s, g.start, i0);
    rest = slot8(p, s, g.start, i0 + 1);
  }
  const int64_t slot = (int64_t)p.rows_per_tile * (D + 4);
  // Every warp waits, those with nothing to join too: this grid must not be complete before the other is.
  pdl_wait_prior();
  if (n < 2) return;  // an empty request, or a unit that one CTA finished: written by the attention kernel

  float m = -INFINITY, l = 0.f, a[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) a[c] = 0.f;
#pragma unroll 1
  for (int j0 = 0; j0 < n; j0 += kFlight) {
    // (m, l) one state per lane, a[] all lanes of one state after the other
    const int own = j0 + (lane & (kFlight - 1));
    float2 st = make_float2(-INFINITY, 0.f);
    if (own < n) st = __ldcg(reinterpret_cast<const float2*>(own == 0 ? first : rest + (int64_t)(own - 1) * 2 * slot) + r);
    float v[kFlight][CPL];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int i = min(j0 + j, n - 1);
      const float* x = (i == 0 ? first : rest + (int64_t)(i - 1) * 2 * slot) + 4 * p.rows_per_tile + r * D + lane * CPL;
      if (CPL == 4) {
        const float4 q = __ldcg(reinterpret_cast<const float4*>(x));
        v[j][0] = q.x;
        v[j][1] = q.y;
        v[j][CPL - 2] = q.z;
        v[j][CPL - 1] = q.w;
      } else {
        const float2 q = __ldcg(reinterpret_cast<const float2*>(x));
        v[j][0] = q.x;
        v[j][1] = q.y;
      }
    }
    float top = st.y != 0.f ? st.x : -INFINITY;  // (l = 0: an empty state)
#pragma unroll
    for (int o = kFlight / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = fmaxf(top, m);
    const float f = m == top ? 1.f : exp2f(m - top);
    m = top;
    const float w = st.y == 0.f ? 0.f : st.x == top ? 1.f : exp2f(st.x - top);
    float lw = w * st.y;
#pragma unroll
    for (int o = kFlight / 2; o; o >>= 1) lw += __shfl_xor_sync(0xffffffffu, lw, o);
    l = fmaf(l, f, lw);
#pragma unroll
    for (int c = 0; c < CPL; ++c) a[c] *= f;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const float wj = __shfl_sync(0xffffffffu, w, j);
      if (j0 + j < n) {
#pragma unroll
        for (int c = 0; c < CPL; ++c) a[c] = fmaf(wj, v[j][c], a[c]);
      }
    }
  }
  if (lane == 0) put_ml8(p, g, r, m, l);
#pragma unroll
  for (int c = 0; c < CPL; ++c) put_a8(p, g, r, lane * CPL + c, l, a[c]);
}

}  // namespace

cudaError_t launch_attn8_join(const Attn8Params& p, cudaStream_t s, bool pdl) {
  const int64_t rows = (int64_t)p.B * p.H_kv * p.R;  // below 2^31 (ss_create)
  const dim3 grid((unsigned)((rows + kWarps - 1) / kWarps)), block(kWarps * 32);
  return launch_kernel(p.d == 128 ? attn8_join_kernel<128> : attn8_join_kernel<64>, grid, block, 0, s, pdl, p);
}

}  // namespace ss
