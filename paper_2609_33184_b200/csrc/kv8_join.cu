// Joins the partial states of units that the attention launch cut (kv8.cuh): a warp per query row, so
// that many states of many rows are read by the whole GPU.  (Joined by the last CTA of each unit instead, with
// a ticket: one launch less and slower everywhere, 9.8 against 7.9 us for one request of 1024 tokens, 52
// against 48 for 131071, 55 against 29 for a round of 2 x 6909 tokens and 40 rows per kv-head.)
//
// Directly behind the attention kernel (decoding) a warp works the shares out again from the lengths, and
// does so before it waits: the attention kernel let this one start only after everything in front of it, the
// lengths' producer too, was complete.  At a round's end, when the lengths' buffer may have been written
// anew, it finds a cut unit's parts where the attention kernel says (put_cut8).  Bound by dependent reads of L2.
#include "kv8.cuh"

namespace ss {
namespace {

constexpr int kWarps = 4;
// States in flight: 16, and 4 where the registers of 16 (three blocks per SM) would keep a window's rows from
// running side by side: many rows mean many units, so few states of each (a round of 16 x 8 candidates over 8192
// tokens 104 us against 106; with few rows 16 are better, 3 x 24 queries over 1000 tokens 10.7 us against 12.0).
constexpr int kFlight = 16, kFlightMany = 4;
bool many_rows(const Attn8Params& p) { return p.window && (int64_t)p.B * p.H_kv * p.R > 3 * kWarps * kNumSM; }
bool few_rows(const Attn8Params& p) { return p.window && p.mode == kCut8 && (int64_t)p.B * p.H_kv * p.R <= 3 * kNumSM; }

// A query row and where its unit's states are: n of them, the first at `first`, the others `step` floats
// apart from `rest`; n = 0: empty request, n = 1: finished by one CTA, not in the scratch area.
struct Row8 {
  Seg8 g;
  int r, rr, rt;            // row in its unit, in its kv-head; row tile
  int n;
  const float *first, *rest;
  int64_t step;
};
// Which row it is (nothing that the kernel in front has to write), and where its states are.
__device__ __forceinline__ Row8 row_at8(const Attn8Params& p, uint32_t row) {
  Row8 w;
  Seg8& g = w.g;
  const uint32_t pair = row / (uint32_t)p.R;
  w.rr = (int)(row - pair * p.R);
  g.b = (int)(pair / (uint32_t)p.H_kv);
  g.kvh = (int)pair - g.b * p.H_kv;
  const int rt = (int)((uint32_t)w.rr / (uint32_t)p.rows_per_tile);
  w.r = w.rr - rt * p.rows_per_tile;
  g.row0 = rt * p.rows_per_tile;
  g.nrows = min(p.rows_per_tile, p.R - g.row0);
  w.rt = rt;
  w.n = 1;
  w.first = w.rest = nullptr;
  w.step = (int64_t)2 * p.row_tiles * p.rows_per_tile * (p.d + 4);
  return w;
}
// Decoding: from the lengths.
__device__ __forceinline__ void row_states8(const Attn8Params& p, Row8& w, int lane) {
  Seg8& g = w.g;
  const uint32_t units = (uint32_t)p.H_kv;
  Share8 s = {};
  const auto tiles = [&](int b) { return tiles8(p.window ? len8<true>(p, b) : len8(p, b)); };
  g.n = tiles(g.b);
  uint32_t sum = 0, before = 0;  // tiles of the requests before this one
  for (int b = lane; b < p.B; b += 32) {
    const uint32_t n = units * tiles(b);
    sum += n;
    if (b < g.b) before += n;
  }
  s.total = __reduce_add_sync(0xffffffffu, sum);
  before = __reduce_add_sync(0xffffffffu, before);
  w.n = 0;
  s.rt = (uint32_t)w.rt;
  if (g.n > 0) {
    set_shares8(p.shares, &s);
    g.start = before + (uint32_t)g.kvh * g.n;
    const int i0 = min((int)share_of8(s, g.start), p.shares - 1);  // (no address depends on more than these two)
    w.n = min((int)share_of8(s, g.start + g.n - 1), p.shares - 1) - i0 + 1;
    w.first = slot8(p, s, g.start, i0);
    w.rest = slot8(p, s, g.start, i0 + 1);
  }
}
// In a round: from what the attention kernel has left in the row's state.
__device__ __forceinline__ void row_states8(const Attn8Params& p, Row8& w, float2 st) {
  if (!(st.y < 0.f)) return;
  // (what an aborted launch leaves may be an older call's: inside the scratch area all the same)
  const uint32_t slot = min((uint32_t)st.x, 2 * (uint32_t)p.shares * p.row_tiles - 1);
  w.n = min((int)-st.y, p.shares - (int)(slot / (2 * (uint32_t)p.row_tiles)));
  w.first = slot_at8(p, slot);
  w.rest = slot_at8(p, 2 * (slot / 2 + p.row_tiles));
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

// Adds states j0 .. n - 1 of the row to (m, l, a); a lane holds D / 32 head dims.
template <int D, int kFlight>
__device__ __forceinline__ void add_states(const Attn8Params& p, const Row8& w, int j0, int n, int lane, float& m, float& l,
                                           float (&a)[D / 32]) {
  constexpr int CPL = D / 32;
#pragma unroll 1
  for (; j0 < n; j0 += kFlight) {
    // (m, l) one state per lane, a[] all lanes of one state after the other
    const int own = j0 + (lane & (kFlight - 1));
    float2 st = make_float2(-INFINITY, 0.f);
    if (own < n)
      st = __ldcg(reinterpret_cast<const float2*>(own == 0 ? w.first : w.rest + (own - 1) * w.step) + w.r);
    float v[kFlight][CPL];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {  // (a row of a window has two or three: loads past the last would be most of them)
      const int i = j0 + j;
      if (i < n)
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
      if (j0 + j < n) {
#pragma unroll
        for (int c = 0; c < CPL; ++c) a[c] = fmaf(wj, v[j][c], a[c]);
      }
    }
  }
}

// All of them.  SPLIT: the block's warps take a quarter each and the first adds what the others have found: one row a
// block, where rows are few and their states many (129 states one after the other took 10 us).  True in the warp that
// has the result.
template <int D, int FLIGHT, bool SPLIT>
__device__ __forceinline__ bool add_all(const Attn8Params& p, const Row8& w, int lane, float& m, float& l,
                                        float (&a)[D / 32]) {
  constexpr int CPL = D / 32;
  if (!SPLIT) {
    add_states<D, FLIGHT>(p, w, 0, w.n, lane, m, l, a);
    return true;
  }
  __shared__ float2 ml_s[kWarps];
  __shared__ float a_s[kWarps][D];
  const int warp = threadIdx.x >> 5, j0 = w.n * warp / kWarps, j1 = w.n * (warp + 1) / kWarps;
  if (warp == 0) {
    add_states<D, FLIGHT>(p, w, j0, j1, lane, m, l, a);
  } else {
    float m1 = -INFINITY, l1 = 0.f, a1[CPL];
#pragma unroll
    for (int c = 0; c < CPL; ++c) a1[c] = 0.f;
    add_states<D, FLIGHT>(p, w, j0, j1, lane, m1, l1, a1);
    if (lane == 0) ml_s[warp] = make_float2(m1, l1);
#pragma unroll
    for (int c = 0; c < CPL; ++c) a_s[warp][lane * CPL + c] = a1[c];
  }
  __syncthreads();
  if (warp) return false;
#pragma unroll
  for (int i = 1; i < kWarps; ++i) {
    const float2 st = ml_s[i];
    if (st.y == 0.f) continue;
    const float top = fmaxf(m, st.x), f = m == top ? 1.f : exp2f(m - top), wt = st.x == top ? 1.f : exp2f(st.x - top);
    m = top;
    l = fmaf(l, f, wt * st.y);
#pragma unroll
    for (int c = 0; c < CPL; ++c) a[c] = fmaf(wt, a_s[i][lane * CPL + c], a[c] * f);
  }
  return true;
}

template <int D, bool ROUND, int FLIGHT, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32) attn8_join_kernel(const __grid_constant__ Attn8Params p) {
  constexpr int CPL = D / 32;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const uint32_t row = SPLIT ? blockIdx.x : blockIdx.x * kWarps + (threadIdx.x >> 5);  // (request, kv-head, row)
  if (row >= (uint32_t)p.B * p.H_kv * p.R) return;  // (the block's first warp has a row)
  Row8 w = row_at8(p, row);
  if (!ROUND) row_states8(p, w, lane);
  // Every warp waits, those with nothing to join too: this grid must not be complete before the other is.
  pdl_wait_prior();
  if (ROUND) row_states8(p, w, __ldcg(p.part_ml + ((int64_t)w.g.b * p.H_kv + w.g.kvh) * p.R_stride + w.rr));
  if (w.n < 2) return;  // written by the attention kernel
  float m = -INFINITY, l = 0.f, a[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) a[c] = 0.f;
  if (!add_all<D, FLIGHT, SPLIT>(p, w, lane, m, l, a)) return;
  if (lane == 0) put_ml8(p, w.g, w.r, m, l);
#pragma unroll
  for (int c = 0; c < CPL; ++c) put_a8(p, w.g, w.r, lane * CPL + c, l, a[c]);
}

// End of a round whose history is one 8-bit chunk: its states, joined or not, and the local segment's
// straight to O and LSE.
template <int D, int FLIGHT, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32) attn8_finalize_kernel(const __grid_constant__ Attn8Params p,
                                                                     const Final8 out) {
  constexpr int CPL = D / 32;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const uint32_t row = SPLIT ? blockIdx.x : blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (row >= (uint32_t)p.B * p.H_kv * p.R) return;
  Row8 w = row_at8(p, row);
  const int64_t at = ((int64_t)w.g.b * p.H_kv + w.g.kvh) * p.R_stride + w.rr;
  pdl_wait_prior();
  float m = -INFINITY, l = 0.f, a[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) a[c] = 0.f;
  // the local segment's state and the row's, if it was finished by one CTA (fetched while that is worked out)
  float2 ml = make_float2(-INFINITY, 0.f);
  float v[CPL], whole[CPL];
  if (out.loc_ml) {
    ml = __ldcg(out.loc_ml + at);
    load_a<CPL>(out.loc_a + at * D + lane * CPL, v);
  }
  const float2 st = __ldcg(p.part_ml + at);
  load_a<CPL>(p.part_a + at * D + lane * CPL, whole);
  row_states8(p, w, st);
  if (ml.y != 0.f && ml.x != -INFINITY) {  // (an identity state's a[] is undefined)
    m = ml.x;
    l = ml.y;
#pragma unroll
    for (int c = 0; c < CPL; ++c) a[c] = v[c];
  }
  if (w.n >= 2) {
    if (!add_all<D, FLIGHT, SPLIT>(p, w, lane, m, l, a)) return;
  } else if (SPLIT && threadIdx.x >= 32) {
    return;
  } else if (w.n == 1 && st.y != 0.f) {
    const float top = fmaxf(m, st.x), f = m == top ? 1.f : exp2f(m - top), wt = st.x == top ? 1.f : exp2f(st.x - top);
    m = top;
    l = fmaf(l, f, wt * st.y);
#pragma unroll
    for (int c = 0; c < CPL; ++c) a[c] = fmaf(wt, whole[c], a[c] * f);
  }
  const bool some = l > 0.f || l != l;
  const float inv = some ? 1.f / l : 0.f;
  __nv_bfloat162* o = reinterpret_cast<__nv_bfloat162*>(out.O + (int64_t)row * D + lane * CPL);
#pragma unroll
  for (int c = 0; c < CPL / 2; ++c) o[c] = __floats2bfloat162_rn(a[2 * c] * inv, a[2 * c + 1] * inv);
  if (out.LSE && lane == 0) out.LSE[row] = some ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

template <int D, int FLIGHT, bool SPLIT>
cudaError_t launch(const Attn8Params& p, const Final8* out, cudaStream_t s, bool pdl) {
  const int64_t rows = (int64_t)p.B * p.H_kv * p.R;  // below 2^31 (ss_create)
  const dim3 grid((unsigned)(SPLIT ? rows : (rows + kWarps - 1) / kWarps)), block(kWarps * 32);
  if (out) return launch_kernel(attn8_finalize_kernel<D, FLIGHT, SPLIT>, grid, block, 0, s, pdl, p, *out);
  auto kernel = p.O ? attn8_join_kernel<D, false, FLIGHT, SPLIT> : attn8_join_kernel<D, true, FLIGHT, SPLIT>;
  return launch_kernel(kernel, grid, block, 0, s, pdl, p);
}
template <int D>
cudaError_t launch_rows(const Attn8Params& p, const Final8* out, cudaStream_t s, bool pdl) {
  if (many_rows(p)) return launch<D, kFlightMany, false>(p, out, s, pdl);
  return few_rows(p) ? launch<D, kFlight, true>(p, out, s, pdl) : launch<D, kFlight, false>(p, out, s, pdl);
}

}  // namespace

cudaError_t launch_attn8_join(const Attn8Params& p, cudaStream_t s, bool pdl) {
  return p.d == 128 ? launch_rows<128>(p, nullptr, s, pdl) : launch_rows<64>(p, nullptr, s, pdl);
}
cudaError_t launch_attn8_finalize(const Attn8Params& p, const Final8& out, cudaStream_t s, bool pdl) {
  return p.d == 128 ? launch_rows<128>(p, &out, s, pdl) : launch_rows<64>(p, &out, s, pdl);
}

}  // namespace ss
