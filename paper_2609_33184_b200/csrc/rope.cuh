// Rotary positions, and rows that join a cache with the rotation on the way.
#pragma once
#include "kv8.cuh"

namespace ss {

constexpr int kRopePairs = 64;   // d / 2 at most
constexpr int kRopeAxes = 4;

struct RopeParams {
  ss_rope rope;              // rot_dim = 0: rows as they are
  uint16_t *Q, *K, *V;       // rows in; Q and V may be null
  int64_t q_sb, q_sh, q_st, k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  uint16_t *Qo, *Ko;         // rotated rows out; Ko null: K and V become tokens of the cache
  int64_t qo_sb, qo_sh, qo_st, ko_sb, ko_sh, ko_st;
  View8 kv;                  // (strides in bytes)
  int bits;                  // of the cache: 16, 8, or 0 without one
  const int32_t* pos;        // [axes, B, T] by input row, or null: off[b] + row of the call
  const int32_t *idx, *cnt, *off;  // each may be null: rows in order, all T of them, from token (position) 0
  int B, H_q, H_kv, T, d;    // H_q = 0 without Q, H_kv = 0 without K
  uint32_t* status;
};
cudaError_t launch_rope(const RopeParams& p, cudaStream_t s, bool pdl);

}  // namespace ss
