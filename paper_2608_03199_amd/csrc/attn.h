// attn.h -- work items, arguments and launchers of the packed attention
// (attn.hip: plan and C ABI; attn_kernels.h: the kernels, compiled once for each
// type by attn_f32.hip, attn_f16.hip and attn_bf16.hip).
#pragma once

#include "attn_plan.h"
#include "enc_common.h"

namespace sieve {

constexpr int kAttnStats = 3;  // of a partial row: maximum, sum of the probabilities as the
                               // second product takes them, and as they were before rounding

struct AttnArgs {
  const AttnItem* items;
  const AttnJoin* joins;
  int32_t nitems;
  sieve_heads q, k, v, o, dout, dq, dk, dv;
  const uint8_t* key_mask;
  const void* bias;
  float* lse;        // written by the forward pass, read by the backward pass
  int32_t G, heads, d, causal;
  uint32_t g_mul;    // division by G (query_of in attn_kernels.h)
  int32_t g_shift;
  int32_t vec;       // every row may be moved in 16-byte pieces, at offsets of 32 bits from
                     // its tile's first
  float scale;
  // bias: table entry i of a head is relative position i - distance - kAttnPad
  int32_t nb, distance, span;
  const int16_t* bucket_of;  // [span]
  const int16_t* range;      // [nb][2]: first entry of a bucket and the one past its last
  void* dbias;
  // workspace
  float* part_o;     // [parts][rows][DP] unnormalised sums, then [parts][rows][kAttnStats]
  float* part_ml;
  float* part_kv;    // [parts][dk, dv][kAttnKeys][DP]
  float* dsum;       // [queries][heads]: the rows' sums of dout * o
  float* part_bias;  // [kv_heads][row tiles][G][nb]
  float* part_max;   // [kv_heads][row tiles]: the largest |dS| (16-bit floats only)
  int32_t row_tiles;
};

enum AttnKind {
  kAttnFwd, kAttnFwdFew, kAttnJoin, kAttnJoinFew, kAttnDq, kAttnDkv, kAttnDkvJoin
};

// Launch one pass; dp is the padded head size (32, 64, 96 or 128), grid the number of
// work-groups.
hipError_t attn_launch_f32(AttnKind kind, int dp, const AttnArgs& a, int grid, hipStream_t s);
hipError_t attn_launch_f16(AttnKind kind, int dp, const AttnArgs& a, int grid, hipStream_t s);
hipError_t attn_launch_bf16(AttnKind kind, int dp, const AttnArgs& a, int grid, hipStream_t s);

}  // namespace sieve
