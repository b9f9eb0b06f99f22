// 8-bit KV cache: format, addressing, and how attention over it is shared out and joined.
//
// Row format.  A row (one token of one kv-head, d bf16 values) is d codes in e4m3 and one byte
// e + 127, e = the smallest integer in [-32, 80] with max|x| <= 448 * 2^e over the row's finite
// values; the value of a code is code * 2^e.  Powers of two make every scaling exact, so the one
// rounding is that to e4m3 (half a step: 2^-4 of the value, or 2^-10 * 2^e for the smallest);
// since e4m3 is a float format nothing is lost by not using the exact maximum.  The range of e
// keeps the ratio of two scales below 2^112, so that sums of weights and of weights times scales
// stay in fp32's range under one reference.  A byte outside it (a buffer that nobody wrote) counts as the
// nearer end: taken as it is, a row of zeros with byte 0 would enter a row sum with the factor 2^127.
//
// Sharing out.  A unit is one (request, kv-head); its history is cut into tiles of kTok8 tokens.  The
// tiles of all units laid end to end (request by request, lengths read on the device) are given to the
// CTAs in equal shares, so a long request is split over many CTAs and short ones are gathered in one,
// whatever the batch looks like and without the host knowing the lengths.  Where the rows of a unit take
// several row tiles, as many CTAs side by side go through one share, a row tile each: they read the same
// K/V at about the same time, from memory once (laid end to end as units of their own, each row tile
// read it again: 16 x 16384 tokens with 64 rows 201 us against 186, a 320-row tree 960 against 825;
// today 174 and 772).
// A unit inside one share is finished by its CTA; a unit cut by a share's end leaves one partial state
// (m, l, a[d]) per CTA in the scratch area, and a second kernel joins them in CTA order (kv8_join.cu), so
// results do not depend on timing.
#pragma once
#include <cuda_fp16.h>

#include "ss_internal.h"

namespace ss {

constexpr int kTok8 = 128;                 // tokens per tile
constexpr int kCtas8 = 2 * kNumSM;         // CTAs of an attention launch,
constexpr int kCtasFew8 = 3 * kNumSM;      // and at head dim 64 with at most kFew8 rows per row tile
constexpr int kFew8 = 16;
constexpr int kRows8 = 32;                 // most rows of a row tile
constexpr int kMinRows8 = 8;               // rows of a row tile in the CUDA-core kernel
constexpr int kMinExp8 = -32, kMaxExp8 = 80;

// A cache as the kernels address it; all strides in bytes.
struct View8 {
  uint8_t *K, *V, *Ks, *Vs;
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  int64_t ks_sb, ks_sh, ks_st, vs_sb, vs_sh, vs_st;
  const int32_t* page_table;  // null: dense, the outer index is the request
  int n_outer, page_size, pages_per_req;
  int room;                   // tokens a request can hold
  int page_log2;              // log2(page_size), -1 when it is no power of two
  // the same for the tensor-core kernel, which would spend a microsecond on the divisions
  int page_shift;             // pages smaller than a tile: log2(page_size); else -1
  int page_tiles;             // larger pages: tiles per page (1 for the rest)
};

struct Attn8Params {
  const __nv_bfloat16* Q;
  int64_t q_sb, q_sh, q_st;
  View8 kv;
  const int32_t* valid_len;   // device [B] or null (= room)
  int B, H_kv, G, T_q, R, d;
  int row_tiles, rows_per_tile;
  float scale_log2;
  int shares;                 // most shares; the attention launch has shares * row_tiles CTAs
  float* scratch;             // 2 slots per CTA of rows_per_tile * (d + 4) floats: (m, l) pairs, room, a[]
  uint32_t* plan;             // [B + 1] or null: receives the tiles before each request (all kv-heads), and their total
  __nv_bfloat16* O;           // either the finished output ...
  float* LSE;
  float2* part_ml;            // ... or (O null) one partial state per row, as the chunk kernels leave them
  float* part_a;
  int R_stride;
  uint32_t* status;
};

struct Final8 {               // end of a round
  const float2* loc_ml;       // the local segment's states, null without one
  const float* loc_a;
  __nv_bfloat16* O;
  float* LSE;                 // may be null
};

struct Copy8Params {          // write (bf16 -> cache) and read (cache -> bf16)
  uint16_t *K, *V;            // bf16 side
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  View8 kv;
  const int32_t *idx, *cnt, *off;  // each may be null: rows in order, all T of them, from token 0
  int B, H_kv, T, d;
  uint32_t* status;
};

cudaError_t launch_kv8_write(const Copy8Params& p, cudaStream_t s, bool pdl);
cudaError_t launch_kv8_read(const Copy8Params& p, cudaStream_t s, bool pdl);
cudaError_t launch_attn8_simt(const Attn8Params& p, cudaStream_t s, bool pdl);
cudaError_t launch_attn8_tc(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl);
cudaError_t launch_attn8_join(const Attn8Params& p, bool from_plan, cudaStream_t s, bool pdl);
cudaError_t launch_attn8_finalize(const Attn8Params& p, const Final8& out, cudaStream_t s, bool pdl);
cudaError_t attn8_tc_prepare();  // one-time function attributes

// ---- device side ---------------------------------------------------------------------------
__device__ __forceinline__ float pow2_8(int e) { return __int_as_float((e + 127) << 23); }  // |e| <= 126
__device__ __forceinline__ float scale8(uint32_t byte) { return __int_as_float((int)(byte << 23)); }  // 2^(byte - 127)
__device__ __forceinline__ uint32_t byte8(uint32_t byte) { return min(max(byte, (uint32_t)(kMinExp8 + 127)), (uint32_t)(kMaxExp8 + 127)); }

// Length of a request in tokens, clamped to [0, room] (find_share8 reports one outside).
__device__ __forceinline__ int len8(const Attn8Params& p, int b) {
  if (!p.valid_len) return p.kv.room;
  const int v = p.valid_len[b];
  return max(0, min(v, p.kv.room));
}
__device__ __forceinline__ int tiles8(int len) { return (len + kTok8 - 1) / kTok8; }

// Outer index of the page that holds token tok of request b (-1: no such page).
__device__ __forceinline__ int outer8(const View8& kv, int b, int tok, int* inner) {
  if (!kv.page_table) {
    *inner = tok;
    return b;
  }
  const int pg = tok / kv.page_size;
  *inner = tok - pg * kv.page_size;
  const int id = kv.page_table[(int64_t)b * kv.pages_per_req + pg];
  return (id < 0 || id >= kv.n_outer) ? -1 : id;
}

// A CTA's share of all tiles, and the walk through its segments (a segment = the part of one unit
// that lies in the share).  Tiles are numbered in 32 bits: the host sees to it that all rooms together
// hold fewer than 2^31.  The first `more` shares have q + 1 tiles, the others q.
struct Share8 {
  uint32_t total, lo, hi;   // tiles of the launch; this CTA's range
  uint32_t ctas, q, more;   // shares
  uint32_t idx, rt;         // this CTA's share and row tile
  uint32_t b0, base0;       // request that holds tile `lo`, and the tiles before it
};
__device__ __forceinline__ uint32_t share_lo8(const Share8& s, uint32_t i) { return i * s.q + min(i, s.more); }
// The share that holds tile x.
__device__ __forceinline__ uint32_t share_of8(const Share8& s, uint32_t x) {
  const uint32_t big = s.more * (s.q + 1);
  return x < big ? x / (s.q + 1) : s.more + (x - big) / s.q;
}

// From the number of tiles to at most `most` shares.
__device__ __forceinline__ void set_shares8(uint32_t most, Share8* s) {
  s->ctas = min(max(s->total, 1u), most);
  s->q = s->total / s->ctas;
  s->more = s->total - s->q * s->ctas;
}

// Tiles (all kv-heads) of requests b0 + 4 * lane .. + 3: 128 requests per step of a warp, whose loads go
// out together.
__device__ __forceinline__ uint32_t tiles_of_four8(const Attn8Params& p, int b0, uint32_t (&n)[4], bool* bad) {
  const uint32_t units = (uint32_t)p.H_kv;
  const int b = b0 + 4 * (threadIdx.x & 31);
  int len[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) len[j] = b + j >= p.B ? 0 : p.valid_len ? p.valid_len[b + j] : p.kv.room;
  uint32_t sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    *bad |= len[j] < 0 || len[j] > p.kv.room;
    n[j] = units * tiles8(max(0, min(len[j], p.kv.room)));
    sum += n[j];
  }
  return sum;
}
__device__ __forceinline__ uint32_t warp_scan8(uint32_t v) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += up;
  }
  return v;
}

// By one whole warp.  CTA 0 also reports lengths that had to be clamped.
__device__ __forceinline__ Share8 find_share8(const Attn8Params& p) {
  const int lane = threadIdx.x & 31;
  Share8 s = {};
  uint32_t n[4], sum = 0, mine = 0;
  bool bad = false;
#pragma unroll 1
  for (int b = 0; b < p.B; b += 128) sum += mine = tiles_of_four8(p, b, n, &bad);
  if (blockIdx.x == 0 && __any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, SS_DEV_BAD_VALID_LEN);
  s.total = __reduce_add_sync(0xffffffffu, sum);
  s.idx = blockIdx.x;
  if (p.row_tiles > 1) {
    s.idx /= (uint32_t)p.row_tiles;
    s.rt = blockIdx.x - s.idx * p.row_tiles;
  }
  set_shares8(p.shares, &s);
  if (s.idx >= s.ctas || s.total == 0) return s;
  s.lo = share_lo8(s, s.idx);
  s.hi = share_lo8(s, s.idx + 1);
  uint32_t base = 0;
#pragma unroll 1
  for (int b = 0; b < p.B; b += 128) {
    if (p.B > 128) mine = tiles_of_four8(p, b, n, &bad);  // (else still there)
    const uint32_t incl = warp_scan8(mine);
    const unsigned past = __ballot_sync(0xffffffffu, base + incl > s.lo);
    if (past) {
      // the first lane past the share's start, and which of its four requests
      uint32_t before = base + incl - mine;
      int j = 0;
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (j == k && before + n[k] <= s.lo) {
          before += n[k];
          ++j;
        }
      }
      const int at = __ffs(past) - 1;
      s.b0 = b + 4 * at + __shfl_sync(0xffffffffu, j, at);
      s.base0 = __shfl_sync(0xffffffffu, before, at);
      break;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  return s;
}

struct Seg8 {
  int b, kvh;
  int t0, t1, n;            // tiles [t0, t1) of the unit's n
  int len;                  // tokens of the request
  uint32_t base, start, pos;  // tiles before the request, before the unit, before the segment's end
  int row0, nrows;
};
__device__ __forceinline__ void seg_set8(const Attn8Params& p, const Share8& s, Seg8* g) {
  const uint32_t u = (g->pos - g->base) / (uint32_t)g->n;
  g->kvh = (int)u;
  g->start = g->base + u * g->n;
  g->t0 = (int)(g->pos - g->start);
  g->pos = min(g->start + g->n, s.hi);
  g->t1 = (int)(g->pos - g->start);
  g->row0 = (int)s.rt * p.rows_per_tile;
  g->nrows = min(p.rows_per_tile, p.R - g->row0);
}
__device__ __forceinline__ bool seg_first8(const Attn8Params& p, const Share8& s, Seg8* g) {
  if (s.lo >= s.hi) return false;
  g->b = s.b0;
  g->len = len8(p, g->b);
  g->n = tiles8(g->len);
  g->pos = s.lo;
  g->base = s.base0;
  seg_set8(p, s, g);
  return true;
}
__device__ __forceinline__ bool seg_next8(const Attn8Params& p, const Share8& s, Seg8* g) {
  if (g->pos >= s.hi) return false;
  const uint32_t units = (uint32_t)p.H_kv;
#pragma unroll 1
  while (g->pos >= g->base + units * g->n) {  // the next request with tokens (there is one: pos < hi <= total)
    g->base += units * g->n;
    ++g->b;
    g->len = len8(p, g->b);
    g->n = tiles8(g->len);
  }
  seg_set8(p, s, g);
  return true;
}

// Where a finished row goes: O and LSE, or a partial state.  `m` in the base-2 domain.  The state of a row that is
// NaN keeps a finite reference, 0: merges take the maximum of the references and drop states at -inf.
__device__ __forceinline__ void put_ml8(const Attn8Params& p, const Seg8& g, int r, float m, float l) {
  const bool some = l > 0.f || l != l;
  if (p.O) {
    if (p.LSE)
      p.LSE[((int64_t)g.b * p.H_kv + g.kvh) * p.R + g.row0 + r] =
          some ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  } else {
    p.part_ml[((int64_t)g.b * p.H_kv + g.kvh) * p.R_stride + g.row0 + r] = make_float2(l != l ? 0.f : some ? m : -INFINITY, l);
  }
}
__device__ __forceinline__ void put_a8(const Attn8Params& p, const Seg8& g, int r, int c, float l, float a) {
  if (p.O) {
    const float inv = (l > 0.f || l != l) ? 1.f / l : 0.f;
    p.O[(((int64_t)g.b * p.H_kv + g.kvh) * p.R + g.row0 + r) * p.d + c] = __float2bfloat16_rn(a * inv);
  } else {
    p.part_a[(((int64_t)g.b * p.H_kv + g.kvh) * p.R_stride + g.row0 + r) * p.d + c] = a;
  }
}
// Requests without a visible token, by `n` threads of every CTA.  (Out of line, not unrolled: what a
// kernel seldom runs should not stand between the parts that it always runs.)
static __device__ __noinline__ void put_empty8(const Attn8Params& p, int tid, int n) {
#pragma unroll 1
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    if (len8(p, b) > 0) continue;
    const int rows = p.H_kv * p.R;
#pragma unroll 1
    for (int i = tid; i < rows; i += n) {
      const int kvh = i / p.R, r = i - kvh * p.R;
      if (!p.O) p.part_ml[((int64_t)b * p.H_kv + kvh) * p.R_stride + r] = make_float2(-INFINITY, 0.f);
      else if (p.LSE) p.LSE[(int64_t)b * rows + i] = -INFINITY;
    }
    if (!p.O) continue;
    uint4* o = reinterpret_cast<uint4*>(p.O + (int64_t)b * rows * p.d);  // 8 values of bf16 zeros
#pragma unroll 1
    for (int i = tid; i < rows * (p.d / 8); i += n) o[i] = make_uint4(0, 0, 0, 0);
  }
}

// The record of the lengths that this launch went by, for a join that runs later: by one warp of the
// last CTA, which has the least to do.
static __device__ __noinline__ void put_plan8(const Attn8Params& p) {
  const int lane = threadIdx.x & 31;
  uint32_t base = 0, n[4];
  bool bad = false;
#pragma unroll 1
  for (int b = 0; b < p.B; b += 128) {
    const uint32_t mine = tiles_of_four8(p, b, n, &bad), incl = warp_scan8(mine);
    uint32_t before = base + incl - mine;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (b + 4 * lane + j < p.B) p.plan[b + 4 * lane + j] = before;
      before += n[j];
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) p.plan[p.B] = base;
}

// Slot of share i's state of the unit that begins at tile `start` (in row tile s.rt): the first segment
// of a share uses the even slot of its CTA, a later one (always the last) the odd slot.
__device__ __forceinline__ float* slot8(const Attn8Params& p, const Share8& s, uint32_t start, uint32_t i) {
  const int odd = share_lo8(s, i) < start ? 1 : 0;
  return p.scratch + (int64_t)(2 * (i * p.row_tiles + s.rt) + odd) * p.rows_per_tile * (p.d + 4);
}

}  // namespace ss
