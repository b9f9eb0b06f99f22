// Joins the partial states of units that the attention launch cut (kv8.cuh): a warp per query row, so
// that many states of many rows are read by the whole GPU.  (Joined by the last CTA of each unit instead, with
// a ticket: one launch less and slower everywhere, 9.8 against 7.9 us for one request of 1024 tokens, 52
// against 48 for 131071, 55 against 29 for a round of 2 x 6909 tokens and 40 rows per kv-head.)
//
// Directly behind the attention kernel (decoding) a warp works the shares out again from the lengths, and
// does so before it waits: the attention kernel let this one start only after everything in front of it, the
// lengths' producer too, was complete.  At a round's end, when the lengths' buffer may have been written
// anew, it reads the attention kernel's own record of them.  Bound by dependent reads of L2.
#include "kv8.cuh"

namespace ss {
namespace {

constexpr int kWarps = 4;
constexpr int kFlight = 16;  // states in flight

// A query row and where its unit's states are: n of them, the first at `first`, the others `step` floats
// apart from `rest`; n = 0: empty request, n = 1: finished by one CTA, not in the scratch area.
struct Row8 {
  Seg8 g;
  int r, rr;                // row in its unit, in its kv-head
  int n;
  const float *first, *rest;
  int64_t step;
};
template <bool PLAN>
__device__ __forceinline__ Row8 row8(const Attn8Params& p, int64_t row, int lane) {
  Row8 w;
  Seg8& g = w.g;
  const int pair = (int)(row / p.R);
  w.rr = (int)(row - (int64_t)pair * p.R);
  g.b = pair / p.H_kv;
  g.kvh = pair - g.b * p.H_kv;
  const int rt = w.rr / p.rows_per_tile;
  w.r = w.rr - rt * p.rows_per_tile;
  g.row0 = rt * p.rows_per_tile;
  g.nrows = min(p.rows_per_tile, p.R - g.row0);
  const uint32_t units = (uint32_t)p.H_kv;
  Share8 s = {};
  uint32_t before = 0;  // tiles of the requests before this one
  if (PLAN) {
    before = __ldcg(&p.plan[g.b]);
    g.n = (int)((__ldcg(&p.plan[g.b + 1]) - before) / units);
    s.total = __ldcg(&p.plan[p.B]);
  } else {
    g.n = tiles8(len8(p, g.b));
    uint32_t sum = 0;
    for (int b = lane; b < p.B; b += 32) {
      const uint32_t n = units * tiles8(len8(p, b));
      sum += n;
      if (b < g.b) before += n;
    }
    s.total = __reduce_add_sync(0xffffffffu, sum);
    before = __reduce_add_sync(0xffffffffu, before);
  }
  w.n = 0;
  w.first = w.rest = nullptr;
  w.step = (int64_t)2 * p.row_tiles * p.rows_per_tile * (p.d + 4);
  s.rt = (uint32_t)rt;
  if (g.n > 0) {
    set_shares8(p.shares, &s);
    g.start = before + (uint32_t)g.kvh * g.n;
    const int i0 = min((int)share_of8(s, g.start), p.shares - 1);  // (no address depends on more than these two)
    w.n = min((int)share_of8(s, g.start + g.n - 1), p.shares - 1) - i0 + 1;
    w.first = slot8(p, s, g.start, i0);
    w.rest = slot8(p, s, g.start, i0 + 1);
  }
  return w;
}

template <int CPL>
__device__ __forceinline__ void load_a(const float* x, float (&v)[CPL]) {
  if (CPL == 4) {
    const float4 q = __ldcg(reinterpret_cast<const float4*>(x));
    v[0] = q.x;
    v[1] = q.y;
    v[CPL - 2] = q.z;
    v[CPL - 1] = q.w;
  } else {
    const float2 q = __ldcg(reinterpret_cast<const float2*>(x));
    v[0] = q.x;
    v[1] = q.y;
  }
}

// Adds the row's n states to (m, l, a); a lane holds D / 32 head dims.
template <int D>
__device__ __forceinline__ void add_states(const Attn8Params& p, const Row8& w, int lane, float& m, float& l,
                                           float (&a)[D / 32]) {
  constexpr int CPL = D / 32;
#pragma unroll 1
  for (int j0 = 0; j0 < w.n; j0 += kFlight) {
    // (m, l) one state per lane, a[] all lanes of one state after the other
    const int own = j0 + (lane & (kFlight - 1));
    float2 st = make_float2(-INFINITY, 0.f);
    if (own < w.n)
      st = __ldcg(reinterpret_cast<const float2*>(own == 0 ? w.first : w.rest + (own - 1) * w.step) + w.r);
    float v[kFlight][CPL];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int i = min(j0 + j, w.n - 1);
      load_a<CPL>((i == 0 ? w.first : w.rest + (i - 1) * w.step) + 4 * p.rows_per_tile + w.r * D + lane * CPL, v[j]);
    }
    float top = st.y != 0.f ? st.x : -INFINITY;  // (l = 0: an empty state)
#pragma unroll
    for (int o = kFlight / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = fmaxf(top, m);
    const float f = m == top ? 1.f : exp2f(m - top);
    m = top;
    const float wt = st.y == 0.f ? 0.f : st.x == top ? 1.f : exp2f(st.x - top);
    float lw = wt * st.y;
#pragma unroll
    for (int o = kFlight / 2; o; o >>= 1) lw += __shfl_xor_sync(0xffffffffu, lw, o);
    l = fmaf(l, f, lw);
#pragma unroll
    for (int c = 0; c < CPL; ++c) a[c] *= f;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const float wj = __shfl_sync(0xffffffffu, wt, j);
      if (j0 + j < w.n) {
#pragma unroll
        for (int c = 0; c < CPL; ++c) a[c] = fmaf(wj, v[j][c], a[c]);
      }
    }
  }
}

template <int D, bool PLAN>
__global__ void __launch_bounds__(kWarps * 32) attn8_join_kernel(const __grid_constant__ Attn8Params p) {
  constexpr int CPL = D / 32;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);  // (request, kv-head, row)
  if (row >= (int64_t)p.B * p.H_kv * p.R) return;  // (the block's first warp has a row)
  if (PLAN) pdl_wait_prior();
  const Row8 w = row8<PLAN>(p, row, lane);
  // Every warp waits, those with nothing to join too: this grid must not be complete before the other is.
  if (!PLAN) pdl_wait_prior();
  if (w.n < 2) return;  // written by the attention kernel
  float m = -INFINITY, l = 0.f, a[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) a[c] = 0.f;
  add_states<D>(p, w, lane, m, l, a);
  if (lane == 0) put_ml8(p, w.g, w.r, m, l);
#pragma unroll
  for (int c = 0; c < CPL; ++c) put_a8(p, w.g, w.r, lane * CPL + c, l, a[c]);
}

// End of a round whose history is one 8-bit chunk: its states, joined or not, and the local segment's
// straight to O and LSE.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) attn8_finalize_kernel(const __grid_constant__ Attn8Params p,
                                                                     const Final8 out) {
  constexpr int CPL = D / 32;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (row >= (int64_t)p.B * p.H_kv * p.R) return;
  pdl_wait_prior();
  const int64_t pair = row / p.R, at = pair * p.R_stride + (row - pair * p.R);
  float m = -INFINITY, l = 0.f, a[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) a[c] = 0.f;
  // the local segment's state (fetched while the unit's place is worked out)
  float2 ml = make_float2(-INFINITY, 0.f);
  float v[CPL];
  if (out.loc_ml) {
    ml = __ldcg(out.loc_ml + at);
    load_a<CPL>(out.loc_a + at * D + lane * CPL, v);
  }
  const Row8 w = row8<true>(p, row, lane);
  if (ml.y != 0.f && ml.x != -INFINITY) {  // (an identity state's a[] is undefined)
    m = ml.x;
    l = ml.y;
#pragma unroll
    for (int c = 0; c < CPL; ++c) a[c] = v[c];
  }
  if (w.n >= 2) {
    add_states<D>(p, w, lane, m, l, a);
  } else if (w.n == 1) {
    const float2 st = __ldcg(p.part_ml + at);
    if (st.y != 0.f) {
      load_a<CPL>(p.part_a + at * D + lane * CPL, v);
      const float top = fmaxf(m, st.x), f = m == top ? 1.f : exp2f(m - top), wt = st.x == top ? 1.f : exp2f(st.x - top);
      m = top;
      l = fmaf(l, f, wt * st.y);
#pragma unroll
      for (int c = 0; c < CPL; ++c) a[c] = fmaf(wt, v[c], a[c] * f);
    }
  }
  const bool some = l > 0.f || l != l;
  const float inv = some ? 1.f / l : 0.f;
  __nv_bfloat162* o = reinterpret_cast<__nv_bfloat162*>(out.O + row * D + lane * CPL);
#pragma unroll
  for (int c = 0; c < CPL / 2; ++c) o[c] = __floats2bfloat162_rn(a[2 * c] * inv, a[2 * c + 1] * inv);
  if (out.LSE && lane == 0) out.LSE[row] = some ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

dim3 join_grid(const Attn8Params& p) {
  const int64_t rows = (int64_t)p.B * p.H_kv * p.R;  // below 2^31 (ss_create)
  return dim3((unsigned)((rows + kWarps - 1) / kWarps));
}

}  // namespace

cudaError_t launch_attn8_join(const Attn8Params& p, bool from_plan, cudaStream_t s, bool pdl) {
  auto kernel = p.d == 128 ? (from_plan ? attn8_join_kernel<128, true> : attn8_join_kernel<128, false>)
                           : (from_plan ? attn8_join_kernel<64, true> : attn8_join_kernel<64, false>);
  return launch_kernel(kernel, join_grid(p), dim3(kWarps * 32), 0, s, pdl, p);
}

cudaError_t launch_attn8_finalize(const Attn8Params& p, const Final8& out, cudaStream_t s, bool pdl) {
  return launch_kernel(p.d == 128 ? attn8_finalize_kernel<128> : attn8_finalize_kernel<64>, join_grid(p), dim3(kWarps * 32),
                       0, s, pdl, p, out);
}

}  // namespace ss
