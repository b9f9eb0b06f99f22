// 8-bit KV cache: format, addressing, and how attention over it is shared out and joined.
//
// Row format.  A row (one token of one kv-head, d bf16 values) is d codes in e4m3 and one byte
// e + 127, e = the smallest integer in [-32, 80] with max|x| <= 448 * 2^e over the row's finite
// values; the value of a code is code * 2^e.  Powers of two make every scaling exact, so the one
// rounding is that to e4m3 (half a step: 2^-4 of the value, or 2^-10 * 2^e for the smallest);
// since e4m3 is a float format nothing is lost by not using the exact maximum.  The range of e
// keeps the ratio of two scales below 2^112, so that sums of weights and of weights times scales
// stay in fp32's range under one reference.
//
// Sharing out.  A unit is one tile of query rows of one (request, kv-head); its history is cut into
// tiles of kTok8 tokens.  The tiles of all units laid end to end (request by request, lengths read
// on the device) are given to the CTAs in equal shares, so a long request is split over many CTAs
// and short ones are gathered in one, whatever the batch looks like and without the host knowing
// the lengths.  A unit inside one share is finished by its CTA; a unit cut by a share's end leaves
// one partial state (m, l, a[d]) per CTA in the scratch area, and the CTA that finishes last (a
// ticket per unit) joins them in CTA order, so the result does not depend on which one that is.
#pragma once
#include <cuda_fp16.h>

#include "ss_internal.h"

namespace ss {

constexpr int kTok8 = 128;                 // tokens per tile
constexpr int kCtas8 = 2 * kNumSM;         // most CTAs of an attention launch
constexpr int kRows8 = 32;                 // most query rows per unit
constexpr int kMinRows8 = 8;               // rows per unit of the CUDA-core kernel
constexpr int kMinExp8 = -32, kMaxExp8 = 80;

// A cache as the kernels address it; all strides in bytes.
struct View8 {
  uint8_t *K, *V, *Ks, *Vs;
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  int64_t ks_sb, ks_sh, ks_st, vs_sb, vs_sh, vs_st;
  const int32_t* page_table;  // null: dense, the outer index is the request
  int n_outer, page_size, pages_per_req;
  int room;                   // tokens a request can hold
};

struct Attn8Params {
  const __nv_bfloat16* Q;
  int64_t q_sb, q_sh, q_st;
  View8 kv;
  const int32_t* valid_len;   // device [B] or null (= room)
  int B, H_kv, G, T_q, R, d;
  int row_tiles, rows_per_tile;
  float scale_log2;
  int min_tiles;              // a share holds at least this many tiles
  float* scratch;             // 2 slots per CTA of rows_per_tile * (d + 2) floats
  unsigned int* tickets;      // one per unit, zero between launches
  __nv_bfloat16* O;           // either the finished output ...
  float* LSE;
  float2* part_ml;            // ... or (O null) one partial state per row, as the chunk kernels leave them
  float* part_a;
  int R_stride;
  uint32_t* status;
};

struct Copy8Params {          // write (bf16 -> cache) and read (cache -> bf16)
  uint16_t *K, *V;            // bf16 side
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  View8 kv;
  const int32_t *idx, *cnt, *off;  // each may be null: rows in order, all T of them, from token 0
  int B, H_kv, T, d;
  uint32_t* status;
};

cudaError_t launch_kv8_write(const Copy8Params& p, cudaStream_t s);
cudaError_t launch_kv8_read(const Copy8Params& p, cudaStream_t s);
cudaError_t launch_attn8_simt(const Attn8Params& p, cudaStream_t s, bool pdl);
cudaError_t launch_attn8_tc(const Attn8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s, bool pdl);
cudaError_t attn8_tc_prepare();  // one-time function attributes

// ---- device side ---------------------------------------------------------------------------
__device__ __forceinline__ float pow2_8(int e) { return __int_as_float((e + 127) << 23); }  // |e| <= 126
__device__ __forceinline__ float scale8(uint32_t byte) { return __int_as_float((int)(byte << 23)); }  // 2^(byte - 127)

// Length of a request in tokens, flagged and clamped when it is outside [0, room].
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

// One CTA's share of all tiles, and the walk through its segments (a segment = the part of one unit
// that lies in the share).
struct Share8 {
  long long total, lo, hi;  // tiles of the launch; this CTA's range
  int ctas;                 // CTAs that have a share
  int b0;                   // request that holds tile `lo`, and the tiles before it
  long long base0;
};
__device__ __forceinline__ long long share_lo8(long long total, int ctas, int i) { return total * i / ctas; }
// The CTA whose share holds tile x: the largest i with floor(total * i / ctas) <= x.
__device__ __forceinline__ int share_of8(long long total, int ctas, long long x) {
  return (int)(((x + 1) * ctas - 1) / total);
}

// By one whole warp.  Lane 0 of CTA 0 also reports lengths that had to be clamped.
__device__ __forceinline__ Share8 find_share8(const Attn8Params& p) {
  const int lane = threadIdx.x & 31;
  const long long units = (long long)p.H_kv * p.row_tiles;
  Share8 s;
  long long sum = 0;
  bool bad = false;
  for (int b = lane; b < p.B; b += 32) {
    sum += tiles8(len8(p, b));
    if (p.valid_len) bad |= p.valid_len[b] < 0 || p.valid_len[b] > p.kv.room;
  }
  if (blockIdx.x == 0 && __any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, SS_DEV_BAD_VALID_LEN);
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  s.total = sum * units;
  const long long want = (s.total + p.min_tiles - 1) / p.min_tiles;
  s.ctas = (int)(want < gridDim.x ? (want > 0 ? want : 1) : gridDim.x);
  s.lo = s.hi = 0;
  s.b0 = 0;
  s.base0 = 0;
  if ((int)blockIdx.x >= s.ctas || s.total == 0) return s;
  s.lo = share_lo8(s.total, s.ctas, blockIdx.x);
  s.hi = share_lo8(s.total, s.ctas, blockIdx.x + 1);
  long long base = 0;
  for (int b = 0; b < p.B; b += 32) {
    long long n = b + lane < p.B ? units * tiles8(len8(p, b + lane)) : 0, incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    const unsigned past = __ballot_sync(0xffffffffu, base + incl > s.lo);
    if (past) {
      const int at = __ffs(past) - 1;
      s.b0 = b + at;
      s.base0 = base + __shfl_sync(0xffffffffu, incl - n, at);
      break;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  return s;
}

struct Seg8 {
  int b, kvh, rt, unit;     // unit = number of the unit among all B * H_kv * row_tiles
  int t0, t1, n;            // tiles [t0, t1) of the unit's n
  int len;                  // tokens of the request
  long long start;          // the unit's first tile among all
  long long pos;            // the segment's end among all tiles
  int row0, nrows;
};
__device__ __forceinline__ void seg_set8(const Attn8Params& p, const Share8& s, long long base, Seg8* g) {
  // (within a request a unit is (kv-head, row tile), row tile fastest: neighbours read the same K/V)
  const int u = (int)((g->pos - base) / g->n);
  g->kvh = u / p.row_tiles;
  g->rt = u - g->kvh * p.row_tiles;
  g->unit = (g->b * p.H_kv + g->kvh) * p.row_tiles + g->rt;
  g->start = base + (long long)u * g->n;
  g->t0 = (int)(g->pos - g->start);
  const long long end = g->start + g->n < s.hi ? g->start + g->n : s.hi;
  g->t1 = (int)(end - g->start);
  g->pos = end;
  g->row0 = g->rt * p.rows_per_tile;
  g->nrows = min(p.rows_per_tile, p.R - g->row0);
}
// Walk: `base` is the number of tiles before request g->b.
__device__ __forceinline__ bool seg_first8(const Attn8Params& p, const Share8& s, long long* base, Seg8* g) {
  if (s.lo >= s.hi) return false;
  g->b = s.b0;
  g->len = len8(p, g->b);
  g->n = tiles8(g->len);
  g->pos = s.lo;
  *base = s.base0;
  seg_set8(p, s, *base, g);
  return true;
}
__device__ __forceinline__ bool seg_next8(const Attn8Params& p, const Share8& s, long long* base, Seg8* g) {
  if (g->pos >= s.hi) return false;
  const long long units = (long long)p.H_kv * p.row_tiles;
  while (g->pos >= *base + units * g->n) {  // the next request with tokens (there is one: pos < hi <= total)
    *base += units * g->n;
    ++g->b;
    g->len = len8(p, g->b);
    g->n = tiles8(g->len);
  }
  seg_set8(p, s, *base, g);
  return true;
}

// Where a finished row goes: O and LSE, or a partial state.  `m` in the base-2 domain.
__device__ __forceinline__ void put_ml8(const Attn8Params& p, const Seg8& g, int r, float m, float l) {
  const bool some = l > 0.f || l != l;
  if (p.O) {
    if (p.LSE)
      p.LSE[((int64_t)g.b * p.H_kv + g.kvh) * p.R + g.row0 + r] =
          some ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  } else {
    p.part_ml[((int64_t)g.b * p.H_kv + g.kvh) * p.R_stride + g.row0 + r] = make_float2(some ? m : -INFINITY, l);
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
// Requests without a visible token, by `n` threads of every CTA.
__device__ __forceinline__ void put_empty8(const Attn8Params& p, int tid, int n) {
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    if (len8(p, b) > 0) continue;
    for (int i = tid; i < p.H_kv * p.R; i += n) {
      const int kvh = i / p.R, r = i - kvh * p.R;
      if (!p.O) p.part_ml[((int64_t)b * p.H_kv + kvh) * p.R_stride + r] = make_float2(-INFINITY, 0.f);
      else if (p.LSE) p.LSE[((int64_t)b * p.H_kv + kvh) * p.R + r] = -INFINITY;
    }
    if (p.O)
      for (int64_t i = tid; i < (int64_t)p.H_kv * p.R * p.d; i += n)
        p.O[(int64_t)b * p.H_kv * p.R * p.d + i] = __float2bfloat16_rn(0.f);
  }
}

template <int N>
__device__ __forceinline__ void bar8() {
  asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
}

// Slot of CTA i's state of the unit that begins at tile `start` (first CTA i0): the first segment of a
// share uses the CTA's even slot, a later one (always the last) the odd slot.
__device__ __forceinline__ float* slot8(const Attn8Params& p, const Share8& s, long long start, int i) {
  const int odd = share_lo8(s.total, s.ctas, i) < start ? 1 : 0;
  return p.scratch + (int64_t)(2 * i + odd) * p.rows_per_tile * (p.d + 2);
}

// sum over the unit's n states of weight * a[c] for ROWS rows from r on, ROWS * STATES loads in flight
template <int D, int ROWS, int STATES, int STEP>
__device__ __forceinline__ void join_rows8(const Attn8Params& p, const Seg8& g, const float* first, const float* rest,
                                           const float2* w, int block, int r0, int r, int n, int c) {
  const int64_t slot = (int64_t)p.rows_per_tile * (D + 2);
  float a[ROWS];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) a[k] = 0.f;
#pragma unroll 1
  for (int j0 = 0; j0 < n; j0 += STATES) {
    float v[STATES][ROWS], f[STATES][ROWS];
#pragma unroll
    for (int j = 0; j < STATES; ++j) {
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        const int row = r + k * STEP;
        f[j][k] = (j0 + j < n && row < block) ? w[(j0 + j) * block + row].x : 0.f;
        v[j][k] = 0.f;
        if (f[j][k] != 0.f) {  // (a state of weight 0 may be unwritten)
          const float* src = j0 + j == 0 ? first : rest + (int64_t)(j0 + j - 1) * 2 * slot;
          v[j][k] = __ldcg(src + 2 * p.rows_per_tile + (r0 + row) * D + c);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < STATES; ++j)
#pragma unroll
      for (int k = 0; k < ROWS; ++k) a[k] = fmaf(f[j][k], v[j][k], a[k]);
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const int row = r + k * STEP;
    if (row < block) put_a8(p, g, r0 + row, c, w[n * block + row].y, a[k]);
  }
}

// By N threads (128 or 256), after each has stored its part of this CTA's state in its slot: takes the
// unit's ticket and, for the last CTA, joins all states.  *flag and buf (kJoinBuf8 pairs) are shared
// memory.  A read of another CTA's state is a read of L2, so all of a block of rows' (m, l) are fetched at once,
// then their a[] with 2048 loads in flight: one row and state after the other, the join
// took 120 us for 37 states of 4 rows.
constexpr int kJoinBuf8 = 512;
static_assert(kCtas8 + 1 <= kJoinBuf8, "a row's states fit the buffer");
template <int D, int N>
__device__ __noinline__ void join8(const Attn8Params& p, const Share8& s, const Seg8& g, int tid, int* flag, float2* buf) {
  const int i0 = share_of8(s.total, s.ctas, g.start), i1 = share_of8(s.total, s.ctas, g.start + g.n - 1);
  __threadfence();
  bar8<N>();
  if (tid == 0) {
    const int last = atomicAdd(&p.tickets[g.unit], 1u) == (unsigned)(i1 - i0);
    if (last) p.tickets[g.unit] = 0;  // nobody else touches it any more in this launch
    *flag = last;
  }
  bar8<N>();
  if (!*flag) return;
  __threadfence();
  const int n = i1 - i0 + 1;               // >= 2: the unit is cut
  const float* first = slot8(p, s, g.start, i0);
  const float* rest = slot8(p, s, g.start, i0 + 1);   // those after the first are the CTAs' even slots
  const int64_t slot = (int64_t)p.rows_per_tile * (D + 2);
  const int most = kJoinBuf8 / (n + 1);  // rows at a time, >= 1: n <= kCtas8
  for (int r0 = 0; r0 < g.nrows; r0 += most) {
    const int block = min(most, g.nrows - r0);
    for (int f = tid; f < n * block; f += N) {
      const int j = f / block, r = f - j * block;
      const float* src = j == 0 ? first : rest + (int64_t)(j - 1) * 2 * slot;
      buf[f] = __ldcg(reinterpret_cast<const float2*>(src) + r0 + r);
    }
    bar8<N>();
    // eight lanes per row: maximum, weights, sum (left in entry n of the row)
    for (int rr = tid >> 3; rr < (block + N / 8 - 1) / (N / 8) * (N / 8); rr += N / 8) {
      const int r = min(rr, block - 1), part = tid & 7;
      const bool mine = rr < block;
      float m = -INFINITY, l = 0.f;
      for (int j = part; j < n; j += 8) {
        const float2 st = buf[j * block + r];
        if (st.y != 0.f) m = fmaxf(m, st.x);
      }
#pragma unroll
      for (int o = 4; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      for (int j = part; j < n; j += 8) {
        const float2 st = buf[j * block + r];
        const float w = st.y == 0.f ? 0.f : st.x == m ? 1.f : exp2f(st.x - m);  // (an empty state's a[] is not read)
        l = fmaf(w, st.y, l);
        if (mine) buf[j * block + r].x = w;
      }
#pragma unroll
      for (int o = 4; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
      if (mine && part == 0) {
        buf[n * block + r].y = l;
        put_ml8(p, g, r0 + r, m, l);
      }
    }
    bar8<N>();
    constexpr int G = N / D;  // rows side by side
    const int c = tid % D, r = tid / D;
    if (block <= 4 * G) {
      join_rows8<D, 4, 2048 / N / 4, G>(p, g, first, rest, buf, block, r0, r, n, c);
    } else {
      for (int k = r; k < block; k += 8 * G) join_rows8<D, 8, 2048 / N / 8, G>(p, g, first, rest, buf, block, r0, k, n, c);
    }
    bar8<N>();
  }
}

}  // namespace ss
