// loss.hip -- softmax cross entropy of hidden states against a table of vectors, without
// keeping the logits, and its gradients.
//
//   s_tv = scale h_t . w_v,  lse_t = log sum_v exp s_tv,  loss_t = lse_t - s_t,target
//   g_tv = (exp(s_tv - lse_t) - [v = target_t]) dloss_t
//   dh_t = scale sum_v g_tv w_v,  dw_v = scale sum_t g_tv h_t
//
// Forward: tiles of logits stay in accumulators, and what leaves a tile is each row's maximum
// and sum of exponentials over its vectors; a second kernel joins them.
//
// Backward: the logits are computed again, a piece of the vocabulary at a time; the piece's g is
// rounded to 16 bits and kept until both gradients' products have read it (a workspace of at most
// 2^27 values, which the last-level cache holds for the most part: beyond 2^19 rows, a piece of the
// rows at a time, too).  dw of the piece is then complete; dh is summed in fp32 over the pieces.
//
// The matrix products are nearly all of it: 2 rows vocab n operations for the loss, 6 for the
// gradients.
//
// 16-bit inputs are multiplied as they are.  32-bit ones come as three bf16 planes whose sum is
// the value (8 bits each, rounded to nearest), six products of planes: what is left out is at most
// 2^-24 of a product, and as often above as below.  2,001 x 7,919 x 515, both passes: 526 us (518
// to 546 in four runs).  With the pairs of planes one after the other they took 580 where a step's
// planes in LDS together took 498.
//
// g is rounded once, to the inputs' type, and what its target has outweighs the rest of its row:
// g_t,target = -(1 - p_t) dloss_t.  A rounding of it would be the same for every token of a
// frequent word and add up over them, so each row is divided by c_t = 1 - p_t first, from a dot
// product of its own: its target's value is then -1, and the others are at most 1 together (or
// less, where 1 - p_t is below what rounding may leave of it: c_t is never less than that).
// dloss_t c_t is a row's exact factor of dh; in dw's product it goes with h, where its rounding is
// another one for each value and column.  binary16 does not have fp32's range: there g is scaled
// by 2^14, and h's factors by a power of two that brings the largest below 1.
//
// Measured, 8,192 rows, 32,768 vectors, 768 values, bf16: forward 420 us; two pieces of 252 for g
// and 430 for the products (both of 412 GFLOP); 1.70 ms with everything, 0.97 PFLOP/s.  12,007 x
// 100,003 x 1,024: 10.5 ms, 0.94 PFLOP/s.  The matrix units are busy 49% of the forward pass's
// time, 38% of g's, 46% of the products'; LDS has no bank conflicts.  2,048 x 2,048 x 768 f16: 74
// us, seven kernels after each other.
#include <math.h>

#include <algorithm>

#include "loss_plan.h"
#include "mm_tile.h"
#include "once_per_device.h"

using namespace sieve;
using namespace sieve::loss;

namespace {

typedef mm_bf16 bf16;
typedef mm_f16 f16;

constexpr double kLog2e = 1.4426950408889634;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kHigh = 8;                  // tiles of m before the next of n, see mm_tile_at
constexpr float kHalfScale = 16384.f;      // what g in binary16 is scaled by
constexpr float kMostHalf = 65504.f;       // binary16's largest value

// A work-group's tile.  A large one has a CU to itself and eight waves; two small ones share it;
// deep ones are as small, with eight waves and more loads on their way, for launches of no more
// than a tile a CU.  2,048 x 2,048 x 8,192 bf16, 256 tiles: deep 87 us, small 105; 8,192^3: large
// 891 us (1,234 TFLOP/s), small 1,027.
// Triple ones are for values of three planes.
template <int BM_, int BN_, int WM_, int WN_, int kStep_, int kStages, int kPlanes_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kThreads = 64 * WM_ * WN_;
  static constexpr int kStep = kStep_, kPlanes = kPlanes_;
  template <typename T, bool kAcrossA, bool kAcrossB>
  using Tile = MmTile<T, BM, BN, kAcrossA, kAcrossB, WM, WN, kStep, kStages, kPlanes>;
  static constexpr int kTileLds = Tile<mm_bf16, false, false>::kLds;
  static constexpr int kLds = kTileLds + WM * BN * 8;  // and the forward pass's parts
  static constexpr uint32_t kMost = kLds > 81920 ? 256 : 512;  // work-groups on the chip
};
typedef Shape<256, 256, 2, 4, 64, 2, 1> Large;
typedef Shape<128, 128, 2, 2, 64, 2, 1> Small;
typedef Shape<128, 128, 2, 4, 64, 4, 1> Deep;
typedef Shape<128, 128, 2, 4, 32, 3, 3> Triple;

struct Targets {
  const void* p;
  int bytes;
  int64_t vocab;
  // the row's vector, or -1
  __device__ __forceinline__ int64_t at(int64_t row) const {
    const int64_t t = bytes == 8 ? ((const int64_t*)p)[row] : (int64_t)((const int32_t*)p)[row];
    return t >= 0 && t < vocab ? t : -1;
  }
};

__device__ __forceinline__ float other_half(float v) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const u32x2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

// The LDS address of what a kernel holds there.
__device__ __forceinline__ uint32_t lds_of(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// Two parts of a row's sum as one.  Differences of dot products are taken before they are scaled: a
// loss near 0 keeps its bits, however large the logits are.
__device__ __forceinline__ Part join(Part a, Part b, float c2) {
  const float top = fmaxf(a.top, b.top);
  const float at = top == -INFINITY ? 0.f : top;
  return {top, a.sum * exp2_of((a.top - at) * c2) + b.sum * exp2_of((b.top - at) * c2)};
}

struct Logits {
  MmOperand w, h;        // a piece of the table; the rows
  int64_t v_first;       // the piece's first vector
  int64_t t_first;       // the rows' first
  int64_t k;             // n, up to the next multiple of 8
  uint32_t tiles_m, tiles_n;
  float c2, c2_rest;     // scale log2(e), and what rounding took from it
  float scale;
  Targets targets;
  // forward
  Part* part;            // [tile of vectors][rows]
  float* target_dot;     // [rows]
  // backward
  const float* lse;
  const Row* row;        // [rows]
  void* g;               // [planes][rows][g_stride]
  int64_t g_stride, g_plane;
};

typedef mm_f32x16 f32x16;

// x = f(x) for the value x of each of the wave's rows' targets that lie among its vectors: `rel`
// from the wave's first, or -1.  There are few: one row at a time, its register found by a number
// that the whole wave knows.
template <int kI, typename F>
__device__ __forceinline__ void each_target(f32x16 (&acc)[kI], int rel, F f) {
  const int half = (int)threadIdx.x >> 5 & 1;
  uint64_t some = __ballot(rel >= 0 && (rel >> 2 & 1) == half);
  while (some) {
    const int lane = __ffsll((unsigned long long)some) - 1;
    some &= some - 1;
    const int v = __builtin_amdgcn_readlane(rel, lane);
    const int r = (v >> 3 & 3) * 4 + (v & 3);
    const bool own = (int)(threadIdx.x & 63) == lane;
#pragma unroll
    for (int i = 0; i < kI; ++i)
      if (v >> 5 == i) acc[i][r] = own ? f(acc[i][r]) : acc[i][r];
  }
}

// The tiles of a launch without splits, in order.
template <typename S>
struct Tiles {
  MmPlaces at;
  uint32_t tiles_m, tiles_n;
  int64_t k;
  __device__ __forceinline__ Tiles(uint32_t tm, uint32_t tn, int64_t k_)
      : at(tm * tn), tiles_m(tm), tiles_n(tn), k(k_) {}
  __device__ __forceinline__ void get(MmWork& w, uint32_t& tm) const {
    uint32_t tn;
    mm_tile_at(at.place, tiles_m, tiles_n, kHigh, tm, tn);
    w = {(int64_t)tm * S::BM, (int64_t)tn * S::BN, 0, k};
  }
  __device__ __forceinline__ bool operator()(MmWork& w) {
    if (!at.there()) return false;
    uint32_t tm;
    get(w, tm);
    at.next();
    return true;
  }
};

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads, 2) void loss_forward_kernel(Logits a) {
  extern __shared__ __attribute__((aligned(1024))) char lds_memory[];
  Part* s_part = (Part*)(lds_memory + S::kTileLds);  // [wave along the vectors][row]
  typedef typename S::template Tile<T, false, false> Tile;
  Tiles<S> ahead(a.tiles_m, a.tiles_n, a.k), tiles = ahead;
  if (!tiles.at.there()) return;
  Tile t(a.w, a.h, 1, lds_of(lds_memory));
  t.start(ahead);
  constexpr int kWave = S::BM / S::WM;   // vectors of a wave
  const int wave_m = Tile::wave() / S::WN, half = (int)threadIdx.x >> 5 & 1;
  for (; tiles.at.there(); tiles.at.next()) {
    MmWork w;
    uint32_t tm;
    tiles.get(w, tm);
    const int64_t first = w.m0 + wave_m * kWave;
    const int left = (int)(a.w.rows - first < kWave ? a.w.rows - first : kWave);
    int rel[Tile::kJ];  // where a row's target lies among the wave's vectors, or -1
#pragma unroll
    for (int j = 0; j < Tile::kJ; ++j) {
      const int64_t row = w.n0 + t.col0 + 32 * j;
      const int64_t v = row < a.h.rows ? a.targets.at(a.t_first + row) : -1;
      const int64_t at = v - a.v_first - first;
      rel[j] = v >= 0 && at >= 0 && at < kWave ? (int)at : -1;
    }
    t.sum(t.steps_of(w), ahead);
#pragma unroll
    for (int j = 0; j < Tile::kJ; ++j) {
      f32x16 acc[Tile::kI];
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < Tile::kI; ++i) {
        acc[i] = t.acc[i][j];
        if (left < kWave) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (Tile::down(i, r) >= left - 4 * half) acc[i][r] = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][r]);
      }
      top = fmaxf(top, other_half(top));
      const float at = top == -INFINITY ? 0.f : top * a.c2;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < Tile::kI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += exp2_of(fmaf(acc[i][r], a.c2, -at));
      sum += other_half(sum);
      // the sum is of 2^(c2 x - at), with at rounded: by as much it is of 2^(c2 (x - top))
      if (top != -INFINITY) sum *= exp2_of(-fmaf(top, a.c2, -at));
      each_target(acc, rel[j], [&](float x) {
        a.target_dot[w.n0 + t.col0 + 32 * j] = x;
        return x;
      });
      if ((threadIdx.x & 32) == 0) s_part[wave_m * S::BN + t.col0 + 32 * j] = Part{top, sum};
    }
    mm_barrier();
    if (threadIdx.x < S::BN && w.n0 + threadIdx.x < a.h.rows) {
      Part p = s_part[threadIdx.x];
#pragma unroll
      for (int i = 1; i < S::WM; ++i) p = join(p, s_part[i * S::BN + threadIdx.x], a.c2);
      a.part[(int64_t)tm * a.h.rows + w.n0 + threadIdx.x] = p;
    }
    // the next tile's first step has a barrier between these reads and the next parts
  }
  t.stop();
}

// Joins the tiles' parts: a work-group takes kRows rows, its 256 / kRows groups of threads every
// so many-th tile of them.
struct Join {
  const Part* part;
  const float* target_dot;
  Targets targets;
  int64_t t_first, rows, tiles;
  float c2, scale;
  float *loss, *lse;
};
template <int kRows>
__global__ __launch_bounds__(256) void loss_join_kernel(Join a) {
  constexpr int kGroups = 256 / kRows;
  __shared__ Part s[kGroups][kRows];
  const int c = threadIdx.x % kRows, g = threadIdx.x / kRows;
  const int64_t row = (int64_t)blockIdx.x * kRows + c;
  Part p{-INFINITY, 0.f};
  if (row < a.rows) {
#pragma unroll 4
    for (int64_t i = g; i < a.tiles; i += kGroups) p = join(p, a.part[i * a.rows + row], a.c2);
  }
  s[g][c] = p;
  __syncthreads();
#pragma unroll
  for (int half = kGroups / 2; half; half /= 2) {
    if (g < half) s[g][c] = p = join(p, s[g + half][c], a.c2);
    __syncthreads();
  }
  if (g != 0 || row >= a.rows) return;
  const float more = log2f(p.sum);
  a.lse[a.t_first + row] = (float)((double)p.top * a.scale + (double)more * 0.6931471805599453);
  if (a.loss)
    a.loss[a.t_first + row] = a.targets.at(a.t_first + row) < 0
                                  ? 0.f
                                  : fmaf(more, kLn2, (p.top - a.target_dot[row]) * a.scale);
}

// ---- few rows ----------------------------------------------------------------------------------
//
// The likelihood of a few rows, say of one token: the table is read once and memory bounds it.
// A wave takes 16 vectors at a time straight from memory into the matrix unit's operands, 16 bytes
// a lane, against the rows (from the cache), and keeps each lane's own largest value and sum.

struct Thin {
  const void *h, *table;
  int64_t h_stride, t_stride, vocab;
  int rows, n;
  float c2;
  Targets targets;
  Part* part;            // [work-group][rows]
  float* target_dot;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t thin_rsrc(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(mm_uniform((char*)const_cast<void*>(p)), 0,
                                           (int)kMmNowhere, 0x00027000);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 thin_mfma(enc_u32x4 a, enc_u32x4 b, f32x4 c, f16) {
  typedef f16 v8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a),
                                                __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 thin_mfma(enc_u32x4 a, enc_u32x4 b, f32x4 c, bf16) {
  typedef bf16 v8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a),
                                                 __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
// 16 values of k: step j multiplies element j of every quarter's operands
__device__ __forceinline__ f32x4 thin_mfma(enc_u32x4 a, enc_u32x4 b, f32x4 c, float) {
  const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
  return c;
}

template <typename F>
__global__ __launch_bounds__(256) void loss_thin_kernel(Thin a) {
  __shared__ Part s_part[4][kThinRows];
  constexpr int kE = 16 / (int)sizeof(F), kStepK = 4 * kE, kAhead = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 15, quarter = lane >> 4;
  const __amdgpu_buffer_rsrc_t hr = thin_rsrc(a.h);
  const uint32_t h_off =
      row < a.rows ? (uint32_t)(row * (uint32_t)a.h_stride) * sizeof(F) : kMmNowhere;
  const int64_t target = row < a.rows ? a.targets.at(row) : -1;
  Part p{-INFINITY, 0.f};
  for (int64_t v0 = ((int64_t)blockIdx.x * 4 + wave) * 16; v0 < a.vocab;
       v0 += (int64_t)gridDim.x * 64) {
    const __amdgpu_buffer_rsrc_t wr = thin_rsrc((const F*)a.table + v0 * a.t_stride);
    const uint32_t w_off =
        v0 + row < a.vocab ? (uint32_t)(row * (uint32_t)a.t_stride) * sizeof(F) : kMmNowhere;
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < a.n; k0 += kAhead * kStepK) {
      enc_u32x4 x[kAhead], y[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = k0 + u * kStepK + quarter * kE;
        // past the end, or the last row: zeros (what is added to kMmNowhere leads nowhere, too)
        const uint32_t wo = k < a.n ? w_off + k * (uint32_t)sizeof(F) : kMmNowhere;
        const uint32_t ho = k < a.n ? h_off + k * (uint32_t)sizeof(F) : kMmNowhere;
        x[u] = __builtin_bit_cast(enc_u32x4,
                                  __builtin_amdgcn_raw_buffer_load_b128(wr, (int)wo, 0, 0));
        y[u] = __builtin_bit_cast(enc_u32x4,
                                  __builtin_amdgcn_raw_buffer_load_b128(hr, (int)ho, 0, 0));
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) c = thin_mfma(x[u], y[u], c, F{});
    }
    // the lane has vectors v0 + 4 quarter .. + 3 of its row
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t v = v0 + 4 * quarter + t;
      if (v < a.vocab) p = join(p, Part{c[t], 1.f}, a.c2);
      if (v == target) a.target_dot[row] = c[t];
    }
  }
#pragma unroll
  for (int o = 16; o < 64; o <<= 1)
    p = join(p, Part{__shfl_xor(p.top, o), __shfl_xor(p.sum, o)}, a.c2);
  if (quarter == 0) s_part[wave][row] = p;
  __syncthreads();
  if (threadIdx.x < a.rows) {
    p = s_part[0][threadIdx.x];
    for (int i = 1; i < 4; ++i) p = join(p, s_part[i][threadIdx.x], a.c2);
    a.part[(int64_t)blockIdx.x * a.rows + threadIdx.x] = p;
  }
}

// The rows' factors, a wave a row, and the largest of them of each work-group.
struct Rows {
  const void *h, *table;
  int64_t h_stride, t_stride, rows;
  int n;
  float scale;
  Targets targets;
  const float *lse, *dloss;
  Row* to;
  float* largest;        // [work-group]
};

template <typename F, int E>
__global__ __launch_bounds__(256) void loss_rows_kernel(Rows a) {
  __shared__ float s[4];
  const int lane = threadIdx.x & 63;
  float largest = 0.f;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows;
       row += (int64_t)gridDim.x * 4) {
    const int64_t target = a.targets.at(row);
    const float d = a.dloss[row];
    Row r{0.f, 0.f};
    if (target >= 0 && d != 0.f) {
      const F* h = (const F*)a.h + row * a.h_stride;
      const F* w = (const F*)a.table + target * a.t_stride;
      float dot = 0.f, size = 0.f;
      for (int col = lane * E; col < a.n; col += 64 * E) {
        if constexpr (E > 1) {
          const EncVec<F, E> x = enc_load<F, E>(h + col), y = enc_load<F, E>(w + col);
#pragma unroll
          for (int j = 0; j < E; ++j) {
            dot = fmaf((float)x.v[j], (float)y.v[j], dot);
            size = fmaf(fabsf((float)x.v[j]), fabsf((float)y.v[j]), size);
          }
        } else {
          dot = fmaf((float)h[col], (float)w[col], dot);
          size = fmaf(fabsf((float)h[col]), fabsf((float)w[col]), size);
        }
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) {
        dot += __shfl_xor(dot, o);
        size += __shfl_xor(size, o);
      }
      const float logit = dot * a.scale, lse = a.lse[row];
      // 1 - p, but no less than what rounding leaves of it, as the row's g may be as much: this sum
      // of n products, and the matrix units' in another order, are each off by up to
      // n 2^-24 sum |h w|, which is far above |logit| where large products cancel.  g is at most 1
      // in any case: of a logit that is infinite, too
      const float least = 0x1p-20f * (4.f + fabsf(logit) + fabsf(lse)) +
                          0x1p-23f * (float)a.n * size * a.scale;
      const float c = fmaxf(-expm1f(logit - lse), fminf(least, 1.f));
      r = {1.f / c, c * d};
    }
    if (lane == 0) a.to[row] = r;
    if (isfinite(r.factor)) largest = fmaxf(largest, fabsf(r.factor));
  }
  if (lane == 0) s[threadIdx.x >> 6] = largest;
  __syncthreads();
  if (threadIdx.x == 0) a.largest[blockIdx.x] = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}

// The power of two next above all of the rows' factors.
__global__ __launch_bounds__(256) void loss_power_kernel(const float* largest, int count,
                                                         int* power) {
  __shared__ float s[4];
  float top = 0.f;
  for (int i = threadIdx.x; i < count; i += 256) top = fmaxf(top, largest[i]);
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    int e = 0;
    frexpf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), &e);
    *power = e;
  }
}

// v as three 8-bit parts, largest first, each rounded to nearest: the second is at most 2^-8 of v,
// the third 2^-17, and their sum is v.  What is not finite is the first part's alone, and what
// would round past the largest value is cut off instead.
__device__ __forceinline__ void split3(float v, bf16 (&p)[3]) {
  const float near = (float)(bf16)v;
  const float cut = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & 0xffff0000u);
  const float a = fabsf(near) == INFINITY ? cut : near;
  const float rest = isfinite(v) ? v - a : 0.f;
  p[0] = (bf16)a;
  p[1] = (bf16)rest;
  p[2] = (bf16)(rest - (float)p[1]);
}

// Rows of n values as the products take them: zeros up to the next multiple of 8, 32-bit values
// as three planes, or 16-bit ones and what rounding took from them as two; with `row` each row
// times its factor (over the power of two), or zeros where it has none.
struct Pack {
  const void* x;
  int64_t stride, rows;
  int n, k;
  void* to;
  int64_t plane;
  int planes;
  const Row* row;
  const int* power;
};

template <typename T>
__global__ __launch_bounds__(256) void loss_pack_kernel(Pack a) {
  typedef std::conditional_t<std::is_same_v<T, float>, bf16, T> U;
  const int per = a.k / 8;
  const int64_t all = a.rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all;
       i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int col = (int)(i % per) * 8;
    float factor = 1.f;
    if (a.row) {
      const Row w = a.row[row];
      factor = w.inverse == 0.f ? 0.f : a.power ? ldexpf(w.factor, -*a.power) : w.factor;
    }
    const T* x = (const T*)a.x + row * a.stride + col;
    constexpr int kPlanes = std::is_same_v<T, float> ? 3 : 2;
    EncVec<U, 8> out[kPlanes];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = col + j < a.n && factor != 0.f ? (float)x[j] * factor : 0.f;
      if constexpr (std::is_same_v<T, float>) {
        bf16 p[3];
        split3(v, p);
#pragma unroll
        for (int q = 0; q < 3; ++q) out[q].v[j] = p[q];
      } else {
        out[0].v[j] = (U)v;
        out[1].v[j] = (U)(v - (float)out[0].v[j]);
      }
    }
#pragma unroll
    for (int q = 0; q < kPlanes; ++q)
      if (q < a.planes) enc_store<U, 8>((U*)a.to + q * a.plane + row * a.k + col, out[q]);
  }
}

// g of a piece: the logits' tiles again, each value turned into its gradient.  F: the inputs'
// type; T: the planes'.
template <typename F, typename T, typename S>
__global__ __launch_bounds__(S::kThreads, 2) void loss_gradient_kernel(Logits a) {
  extern __shared__ __attribute__((aligned(1024))) char lds_memory[];
  typedef typename S::template Tile<T, false, false> Tile;
  Tiles<S> ahead(a.tiles_m, a.tiles_n, a.k), tiles = ahead;
  if (!tiles.at.there()) return;
  Tile t(a.w, a.h, 1, lds_of(lds_memory));
  t.start(ahead);
  constexpr int kWave = S::BM / S::WM;
  const int wave_m = Tile::wave() / S::WN, half = (int)threadIdx.x >> 5 & 1;
  for (; tiles.at.there(); tiles.at.next()) {
    MmWork w;
    uint32_t tm;
    tiles.get(w, tm);
    const int64_t first = w.m0 + wave_m * kWave;
    const int left = (int)(a.w.rows - first < kWave ? a.w.rows - first : kWave);
    int rel[Tile::kJ];
    float inverse[Tile::kJ], lse2[Tile::kJ], rest[Tile::kJ];
#pragma unroll
    for (int j = 0; j < Tile::kJ; ++j) {
      const int64_t row = w.n0 + t.col0 + 32 * j;
      rel[j] = -1;
      inverse[j] = lse2[j] = rest[j] = 0.f;
      if (row < a.h.rows) {
        const int64_t v = a.targets.at(row), at = v - a.v_first - first;
        if (v >= 0 && at >= 0 && at < kWave) rel[j] = (int)at;
        inverse[j] = a.row[row].inverse;
        if constexpr (std::is_same_v<F, f16>) inverse[j] *= kHalfScale;
        // lse in base 2 and the rounding of it and of c2, both by as much as it matters: for
        // logits near lse
        const float lse = a.lse[row];
        const double exact = (double)lse * kLog2e;
        lse2[j] = (float)exact;
        rest[j] = exp2_of(lse / a.scale * a.c2_rest - (float)(exact - (double)lse2[j]));
        if (inverse[j] != 0.f) inverse[j] *= rest[j];
      }
    }
    t.sum(t.steps_of(w), ahead);
#pragma unroll
    for (int j = 0; j < Tile::kJ; ++j) {
      const int64_t row = w.n0 + t.col0 + 32 * j;
      const bool there = row < a.h.rows;
      T* g = (T*)a.g + row * a.g_stride + first + 8 * half;
      f32x16 p[Tile::kI];
#pragma unroll
      for (int i = 0; i < Tile::kI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[i][r] = exp2_of(fmaf(t.acc[i][j][r], a.c2, -lse2[j]));
      each_target(p, rel[j], [&](float x) { return x - 1.f / rest[j]; });
#pragma unroll
      for (int i = 0; i < Tile::kI; ++i) {
        f32x16 x = p[i];
        if (left < kWave) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (Tile::down(i, r) >= left - 4 * half) x[r] = 0.f;
        }
        // a row without a factor gives nothing, whatever it holds
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = inverse[j] == 0.f ? 0.f : x[r] * inverse[j];
        if constexpr (std::is_same_v<F, f16>) {
          // up to 4 times c fit; logits that are good to no more than that give no infinities, but
          // a row that is not a number stays one (its lse is not one, either)
          const float most = fmaf(inverse[j], 0.f, kMostHalf);
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_fmed3f(x[r], -most, most);
        }
        // pairs of 16-bit values; halves of a wave change places so that each lane has 8
        // neighbours
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          constexpr int kPlanes = std::is_same_v<F, float> ? 3 : 1;
          T part[kPlanes][8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if constexpr (kPlanes == 3) {
              T p[3];
              split3(x[8 * q + e], p);
#pragma unroll
              for (int z = 0; z < 3; ++z) part[z][e] = p[z];
            } else {
              part[0][e] = (T)x[8 * q + e];
            }
          }
#pragma unroll
          for (int z = 0; z < kPlanes; ++z) {
            uint32_t d[4];
            __builtin_memcpy(d, part[z], 16);
            const u32x2 lo = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
            const u32x2 hi = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
            const enc_u32x4 out = {lo[0], hi[0], lo[1], hi[1]};
            if (there) *(enc_u32x4*)(g + z * a.g_plane + i * 32 + 16 * q) = out;
          }
        }
      }
    }
  }
  t.stop();
}

// What turns a sum of products into a gradient.
struct Final {
  void* out;               // [rows][n]
  int n;
  float factor;            // scale, over what g was scaled by
  const int* power;        // dtable: the power of two that h was divided by, where it was
  const Row* row;          // dh: the row's own factor; zeros where it has none
};

// A row's factor.
__device__ __forceinline__ float factor_of(const Final& a, int64_t row) {
  if (!a.row) return a.power ? ldexpf(a.factor, *a.power) : a.factor;
  const Row w = a.row[row];
  return w.inverse == 0.f ? 0.f : w.factor * a.factor;
}

// A gradient's product: sums in fp32, [split][rows of m][pitch], or added to what is there; or,
// with final.out, the gradient itself.
struct Product {
  MmOperand a, b;
  int64_t k, per;        // values of k, and of a split
  int planes_b;          // of b, for one of a
  uint32_t tiles_m, tiles_n, splits;
  int64_t rows;          // of m, that are written
  float* out;
  int64_t pitch, split;  // values between rows, and between splits
  int add;
  Final final;
};

// The tiles of a product, split after split.
template <typename S>
struct Splits {
  MmPlaces at;
  uint32_t tiles_m, tiles_n;
  int64_t k, per;
  __device__ __forceinline__ Splits(const Product& a, uint32_t before)
      : at(a.tiles_m * a.tiles_n * a.splits, before), tiles_m(a.tiles_m), tiles_n(a.tiles_n),
        k(a.k), per(a.per) {}
  __device__ __forceinline__ void get(MmWork& w, uint32_t& split) const {
    const uint32_t tiles = tiles_m * tiles_n;
    uint32_t tm, tn;
    split = at.place / tiles;
    mm_tile_at(at.place % tiles, tiles_m, tiles_n, kHigh, tm, tn);
    const int64_t k0 = split * per;
    w = {(int64_t)tm * S::BM, (int64_t)tn * S::BN, k0, k0 + per < k ? k0 + per : k};
  }
  __device__ __forceinline__ bool operator()(MmWork& w) {
    if (!at.there()) return false;
    uint32_t split;
    get(w, split);
    at.next();
    return true;
  }
};

// A work-group's tiles of a product; `before`: the launch's tiles of another one.
template <typename F, typename T, typename S, bool kAcrossA>
__device__ __forceinline__ void run_product(const Product& a, uint32_t before, uint32_t lds) {
  typedef typename S::template Tile<T, kAcrossA, true> Tile;
  Splits<S> ahead(a, before), tiles = ahead;
  if (!tiles.at.there()) return;
  Tile t(a.a, a.b, a.planes_b, lds);
  t.start(ahead);
  for (; tiles.at.there(); tiles.at.next()) {
    MmWork w;
    uint32_t split;
    tiles.get(w, split);
    t.sum(t.steps_of(w), ahead);
    if (a.final.out) {
      const MmPatch<F> to((F*)a.final.out + w.m0 * a.final.n + w.n0, a.final.n, a.rows - w.m0,
                          a.b.rows - w.n0);
      typename MmPatch<F>::Lane lane[Tile::kJ];
#pragma unroll
      for (int j = 0; j < Tile::kJ; ++j) lane[j] = to.lane(t.row0, t.col0 + 32 * j);
#pragma unroll
      for (int i = 0; i < Tile::kI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // rows past the last one are the last one again, and not stored
          const int64_t row = w.m0 + t.row0 + Tile::down(i, r);
          const float factor = factor_of(a.final, row < a.rows ? row : a.rows - 1);
#pragma unroll
          for (int j = 0; j < Tile::kJ; ++j)
            to.store(to.at(lane[j], Tile::down(i, r)),
                     (F)(factor == 0.f ? 0.f : t.acc[i][j][r] * factor));
        }
    } else {
      const MmPatch<float> to(a.out + split * a.split + w.m0 * a.pitch + w.n0, a.pitch,
                              a.rows - w.m0, a.b.rows - w.n0);
#pragma unroll
      for (int j = 0; j < Tile::kJ; ++j) {
        const auto lane = to.lane(t.row0, t.col0 + 32 * j);
#pragma unroll
        for (int i = 0; i < Tile::kI; ++i) {
          f32x16 v = t.acc[i][j];
          if (a.add) {
#pragma unroll
            for (int r = 0; r < 16; ++r) v[r] += to.load(to.at(lane, Tile::down(i, r)));
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) to.store(to.at(lane, Tile::down(i, r)), v[r]);
        }
      }
    }
  }
  t.stop();
}

// Both gradients' products of a piece in one launch: neither's tiles need fill the chip by
// themselves.  8,192 rows, 16,384 vectors, 768 values, bf16: 462 us in large tiles, 511 in small
// ones; one after the other 250 us each.
template <typename F, typename T, typename S>
__global__ __launch_bounds__(S::kThreads, 2) void loss_product_kernel(Product h, Product w) {
  extern __shared__ __attribute__((aligned(1024))) char lds_memory[];
  run_product<F, T, S, false>(h, 0, lds_of(lds_memory));
  mm_barrier();  // the buffers have been read
  run_product<F, T, S, true>(w, h.tiles_m * h.tiles_n * h.splits, lds_of(lds_memory));
}

// The splits' sum as a gradient, 4 values of a row at a time.
struct Finish {
  const float* x;
  int64_t rows, pitch, split;
  int splits;
  Final final;
  int pieces;            // of a row
  int together;          // rows of a work-group
  uint32_t mul;          // index / pieces = (index * mul) >> 32
};

template <typename F>
__global__ __launch_bounds__(256) void loss_finish_kernel(Finish a) {
  for (int64_t first = (int64_t)blockIdx.x * a.together; first < a.rows;
       first += (int64_t)gridDim.x * a.together) {
    const int rows = (int)(a.rows - first < a.together ? a.rows - first : a.together);
    for (int i = threadIdx.x; i < rows * a.pieces; i += 256) {
      const int in = a.pieces == 1 ? i : (int)__umulhi((uint32_t)i, a.mul);
      const int64_t row = first + in;
      const int col = (i - in * a.pieces) * 4;
      const float factor = factor_of(a.final, row);
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      const float* x = a.x + row * a.pitch + col;  // rows are padded to multiples of 8
#pragma unroll 4
      for (int s = 0; s < a.splits; ++s) {
        const EncVec<float, 4> p = enc_load<float, 4>(x + s * a.split);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += p.v[e];
      }
      F* out = (F*)a.final.out + row * a.final.n + col;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < a.final.n) out[e] = (F)(factor == 0.f ? 0.f : v[e] * factor);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------

int check_loss(int64_t rows, int64_t vocab, int32_t n, int32_t dtype) {
  if (!enc_dtype_ok(dtype))
    return set_error(SIEVE_EINVAL, "dtype = %d is not one of SIEVE_F32, SIEVE_F16, SIEVE_BF16",
                     dtype);
  if (rows < 0) return set_error(SIEVE_EINVAL, "rows is negative");
  if (vocab < 1) return set_error(SIEVE_EINVAL, "vocab must be >= 1");
  if (n < 1) return set_error(SIEVE_EINVAL, "n = %d must be >= 1", n);
  if (n > kMaxN) return set_error(SIEVE_EUNSUPPORTED, "n = %d is above %d", n, kMaxN);
  if (rows > kMaxRows || vocab > kMaxRows)
    return set_error(SIEVE_EUNSUPPORTED, "rows or vocab is above %lld", (long long)kMaxRows);
  return SIEVE_OK;
}

int check_call(const void* h, int64_t h_stride, const void* table, int64_t table_stride, int32_t n,
               const void* targets, int32_t target_bytes, float scale, const void* workspace,
               int64_t bytes, int64_t need) {
  if (!h || !table || !targets)
    return set_error(SIEVE_EINVAL, "h, table and targets must be non-NULL");
  if (target_bytes != 4 && target_bytes != 8)
    return set_error(SIEVE_EINVAL, "target_bytes = %d must be 4 or 8", target_bytes);
  if (h_stride < n || table_stride < n)
    return set_error(SIEVE_EINVAL, "a row stride is below n = %d", n);
  if (!(scale > 0.f) || scale == INFINITY)
    return set_error(SIEVE_EINVAL, "scale must be > 0 and finite");
  if (!workspace || bytes < need || ((uintptr_t)workspace & 15))
    return set_error(SIEVE_EINVAL, "workspace must be 16-byte aligned and hold %lld bytes",
                     (long long)need);
  return SIEVE_OK;
}

int blocks_of(int64_t work) { return (int)std::min<int64_t>((work + 255) / 256, 8192); }

template <typename T>
void pack(const void* x, int64_t stride, int64_t rows, int32_t n, int64_t k, void* to,
          int64_t plane, int planes, hipStream_t s, const Row* row = nullptr,
          const int* power = nullptr) {
  const Pack a{x, stride, rows, n, (int)k, to, plane, planes, row, power};
  loss_pack_kernel<T><<<blocks_of(rows * (k / 8)), 256, 0, s>>>(a);
}

template <typename F>
bool rows_aligned(const void* p, int64_t stride) {
  return ((uintptr_t)p & 15) == 0 && (stride * (int64_t)sizeof(F) & 15) == 0;
}

// Whether rows may be multiplied where they lie.
bool direct(const void* p, int64_t stride, int32_t n, int32_t dtype) {
  return dtype != SIEVE_F32 && n % 8 == 0 && stride % 8 == 0 && stride <= kMmMaxStride &&
         ((uintptr_t)p & 15) == 0;
}

// Whether there are few rows, that may be multiplied where they lie.
bool thin(const void* h, int64_t h_stride, const void* table, int64_t t_stride, int64_t rows,
          int32_t n, int size) {
  auto whole = [&](const void* p, int64_t stride) {
    return ((uintptr_t)p & 15) == 0 && stride * size % 16 == 0 && stride <= kMmMaxStride;
  };
  return rows <= (size == 4 ? kThinRows : kThinRows16) && n * size % 16 == 0 &&
         whole(h, h_stride) && whole(table, t_stride);
}

// The operand of rows [0, rows) of x, packed into `to` where that is needed.
template <typename T>
MmOperand operand(const void* x, int64_t stride, int64_t rows, int32_t n, int32_t dtype, int64_t k,
                  void* to, hipStream_t s) {
  if (direct(x, stride, n, dtype)) return {x, stride, rows, 0};
  pack<T>(x, stride, rows, n, k, to, rows * k, dtype == SIEVE_F32 ? 3 : 1, s);
  return {to, k, rows, rows * k};
}

std::atomic<uint64_t> g_large_lds{0};

template <typename K>
hipError_t allow(K* kernel, int bytes) {
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                             bytes);
}

template <typename S>
hipError_t allow_shape() {
  hipError_t r = hipSuccess;
  auto add = [&](auto* kernel) {
    if (r == hipSuccess) r = allow(kernel, S::kLds);
  };
  add(loss_forward_kernel<bf16, S>);
  if constexpr (S::kPlanes == 3) {
    add(loss_gradient_kernel<float, bf16, S>);
    add(loss_product_kernel<float, bf16, S>);
  } else {
    add(loss_forward_kernel<f16, S>);
    add(loss_gradient_kernel<f16, f16, S>);
    add(loss_gradient_kernel<bf16, bf16, S>);
    add(loss_product_kernel<f16, f16, S>);
    add(loss_product_kernel<bf16, bf16, S>);
  }
  return r;
}

int allow_lds() {
  int device = 0;
  ENC_HIP_TRY(hipGetDevice(&device));
  const hipError_t e = once_per_device(g_large_lds, device, [] {
    hipError_t r = allow_shape<Large>();
    if (r == hipSuccess) r = allow_shape<Small>();
    if (r == hipSuccess) r = allow_shape<Deep>();
    return r == hipSuccess ? allow_shape<Triple>() : r;
  });
  ENC_HIP_TRY(e);
  return SIEVE_OK;
}

uint32_t tiles_of(int64_t n, int size) { return (uint32_t)((n + size - 1) / size); }

void join_parts(const Join& a, hipStream_t s) {
  // few rows: more threads for each
  if (a.rows <= 512) loss_join_kernel<4><<<tiles_of(a.rows, 4), 256, 0, s>>>(a);
  else loss_join_kernel<32><<<tiles_of(a.rows, 32), 256, 0, s>>>(a);
}

void set_scale(Logits& a, float scale) {
  const double c2 = (double)scale * kLog2e;
  a.scale = scale;
  a.c2 = (float)c2;
  a.c2_rest = (float)(c2 - (double)a.c2);
}

// f(inputs' type, planes' type)
template <typename F>
void by_type(int32_t dtype, F f) {
  if (dtype == SIEVE_F32) f(float{}, bf16{});
  else if (dtype == SIEVE_F16) f(f16{}, f16{});
  else f(bf16{}, bf16{});
}

template <typename F>
void finish(const float* x, int64_t rows, int64_t pitch, int64_t split, int splits,
            const Final& final, hipStream_t s) {
  Finish a{x, rows, pitch, split, splits, final, (final.n + 3) / 4, 1, 0};
  // some 4 pieces a thread; indexes stay below 2^15, where the multiplier is exact
  a.together = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / a.pieces, rows / 512));
  a.mul = (uint32_t)(((uint64_t(1) << 32) + a.pieces - 1) / a.pieces);
  const int64_t groups = (rows + a.together - 1) / a.together;
  loss_finish_kernel<F><<<(int)std::min<int64_t>(groups, 65536), 256, 0, s>>>(a);
}

// f(the shape), for inputs of type F
template <typename F, typename G>
void by_shape(Size size, G f) {
  if constexpr (std::is_same_v<F, float>) {
    f(Triple{});
  } else {
    if (size == kLarge) f(Large{});
    else if (size == kDeep) f(Deep{});
    else f(Small{});
  }
}

// Sets how a product is cut into tiles and splits.
template <typename S>
void cut(Product& p, int splits) {
  const int64_t each = (p.k + splits - 1) / splits;
  p.per = (each + S::kStep - 1) / S::kStep * S::kStep;
  p.splits = splits;
  p.tiles_m = tiles_of(p.rows, S::BM);
  p.tiles_n = tiles_of(p.final.n, S::BN);
}

}  // namespace

SIEVE_API int64_t sieve_loss_workspace(int64_t rows, int64_t vocab, int32_t n, int32_t dtype,
                                       int32_t backward) {
  clear_error();
  if (int st = check_loss(rows, vocab, n, dtype)) return st;
  if (backward != 0 && backward != 1) return set_error(SIEVE_EINVAL, "backward must be 0 or 1");
  return rows ? layout_of(rows, vocab, n, dtype, backward != 0).bytes : 0;
}

SIEVE_API int sieve_loss_forward(const void* h, int64_t h_stride, const void* table,
                                 int64_t table_stride, int32_t dtype, int64_t rows, int64_t vocab,
                                 int32_t n, const void* targets, int32_t target_bytes, float scale,
                                 float* loss, float* lse, void* workspace, int64_t workspace_bytes,
                                 void* stream) {
  clear_error();
  if (int st = check_loss(rows, vocab, n, dtype)) return st;
  if (rows == 0) return SIEVE_OK;
  const Layout l = layout_of(rows, vocab, n, dtype, false);
  if (int st = check_call(h, h_stride, table, table_stride, n, targets, target_bytes, scale,
                          workspace, workspace_bytes, l.bytes))
    return st;
  if (!lse) return set_error(SIEVE_EINVAL, "lse must be non-NULL");
  if (int st = allow_lds()) return st;
  char* w = (char*)workspace;
  hipStream_t s = (hipStream_t)stream;
  by_type(dtype, [&](auto f, auto t) {
    typedef decltype(f) F;
    typedef decltype(t) T;
    Logits a{};
    set_scale(a, scale);
    a.targets = {targets, target_bytes, vocab};
    a.target_dot = (float*)(w + l.target);
    if (thin(h, h_stride, table, table_stride, rows, n, sizeof(F))) {
      const Thin x{h, table, h_stride, table_stride, vocab, (int)rows, n, a.c2, a.targets,
                   (Part*)(w + l.part), a.target_dot};
      const int groups = (int)std::min<int64_t>((vocab + 63) / 64, kThinMost);
      loss_thin_kernel<F><<<groups, 256, 0, s>>>(x);
      join_parts({x.part, x.target_dot, x.targets, 0, rows, groups, a.c2, scale, loss, lse}, s);
      return;
    }
    a.h = operand<F>(h, h_stride, rows, n, dtype, l.k, w + l.h, s);
    a.k = l.k;
    const MmOperand all_h = a.h;
    // a table that has to be packed is taken in pieces; any is, where a launch would be too large
    const bool as_is = direct(table, table_stride, n, dtype);
    const int64_t piece = as_is ? int64_t(1) << 20 : l.piece;
    for (int64_t t0 = 0; t0 < rows; t0 += kRowChunk) {
      a.h = all_h;
      a.h.p = (const char*)all_h.p + t0 * all_h.stride * 2;
      a.h.rows = std::min(rows - t0, kRowChunk);
      a.t_first = t0;
      const Size size = size_of(std::min(piece, vocab), a.h.rows, l.k, l.planes);
      const int side = kMeasured[size].bm;
      a.tiles_n = tiles_of(a.h.rows, kMeasured[size].bn);
      for (int64_t v0 = 0; v0 < vocab; v0 += piece) {
        const int64_t vs = std::min(piece, vocab - v0);
        a.w = operand<F>((const F*)table + v0 * table_stride, table_stride, vs, n, dtype, l.k,
                         w + l.w, s);
        a.v_first = v0;
        a.tiles_m = tiles_of(vs, side);
        a.part = (Part*)(w + l.part) + v0 / side * a.h.rows;
        by_shape<F>(size, [&](auto shape) {
          typedef decltype(shape) S;
          loss_forward_kernel<T, S>
              <<<mm_grid((uint64_t)a.tiles_m * a.tiles_n, S::kMost), S::kThreads, S::kLds, s>>>(a);
        });
      }
      join_parts({(const Part*)(w + l.part), a.target_dot, a.targets, t0, a.h.rows,
                  tiles_of(vocab, side), a.c2, scale, loss, lse}, s);
    }
  });
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}

SIEVE_API int sieve_loss_backward(const float* dloss, const void* h, int64_t h_stride,
                                  const void* table, int64_t table_stride, int32_t dtype,
                                  int64_t rows, int64_t vocab, int32_t n, const void* targets,
                                  int32_t target_bytes, const float* lse, float scale, void* dh,
                                  void* dtable, void* workspace, int64_t workspace_bytes,
                                  void* stream) {
  clear_error();
  if (int st = check_loss(rows, vocab, n, dtype)) return st;
  hipStream_t s = (hipStream_t)stream;
  const Layout l = layout_of(rows, vocab, n, dtype, true);
  if (rows > 0) {
    if (int st = check_call(h, h_stride, table, table_stride, n, targets, target_bytes, scale,
                            workspace, workspace_bytes, l.bytes))
      return st;
    if (!dloss || !lse) return set_error(SIEVE_EINVAL, "dloss and lse must be non-NULL");
  }
  if (!dh && !dtable) return SIEVE_OK;
  if (rows == 0 && !dtable) return SIEVE_OK;
  if (rows > 0)
    if (int st = allow_lds()) return st;
  char* w = (char*)workspace;
  by_type(dtype, [&](auto f, auto t) {
    typedef decltype(f) F;
    typedef decltype(t) T;
    const Targets tg{targets, target_bytes, vocab};
    const float factor = std::is_same_v<F, f16> ? scale / kHalfScale : scale;
    if (rows == 0) {
      finish<F>(nullptr, vocab, 0, 0, 0, {dtable, n, 0.f, nullptr, nullptr}, s);
      return;
    }
    Row* row = (Row*)(w + l.row);
    // only binary16 needs the power of two
    int* power = std::is_same_v<F, f16> && dtable ? (int*)(w + l.power) : nullptr;
    const Rows r{h, table, h_stride, table_stride, rows, n, scale, tg, lse, dloss, row,
                 (float*)(w + l.largest)};
    const int groups = (int)std::min<int64_t>((rows + 3) / 4, kMostLargest);
    constexpr int kE = 16 / (int)sizeof(F);
    if (n % kE == 0 && rows_aligned<F>(h, h_stride) && rows_aligned<F>(table, table_stride))
      loss_rows_kernel<F, kE><<<groups, 256, 0, s>>>(r);
    else
      loss_rows_kernel<F, 1><<<groups, 256, 0, s>>>(r);
    if (power) loss_power_kernel<<<1, 256, 0, s>>>((const float*)(w + l.largest), groups, power);
    Logits a{};
    const MmOperand all_h = operand<F>(h, h_stride, rows, n, dtype, l.k, w + l.h, s);
    if (dtable)
      pack<F>(h, h_stride, rows, n, l.k, w + l.weighed, rows * l.k, l.weighed_planes, s, row,
              power);
    a.k = l.k;
    set_scale(a, scale);
    a.g = w + l.g;
    a.g_stride = l.piece;
    a.g_plane = l.chunk * l.piece;
    const Size size = size_of(std::min(l.piece, vocab), l.chunk, l.k, l.planes);
    const Final final_h{dh, n, factor, nullptr, row};
    float *sums_h = (float*)(w + l.dh), *sums_w = (float*)(w + l.dw);
    for (int64_t v0 = 0; v0 < vocab; v0 += l.piece) {
      const int64_t vs = std::min(l.piece, vocab - v0);
      a.w = operand<F>((const F*)table + v0 * table_stride, table_stride, vs, n, dtype, l.k,
                       w + l.w, s);
      a.v_first = v0;
      const Final final_w{(F*)dtable + v0 * n, n, factor, power, nullptr};
      for (int64_t t0 = 0; t0 < rows; t0 += l.chunk) {
        const int64_t ts = std::min(l.chunk, rows - t0);
        a.h = all_h;
        a.h.p = (const char*)all_h.p + t0 * all_h.stride * 2;
        a.h.rows = ts;
        a.targets = {(const char*)targets + t0 * target_bytes, target_bytes, vocab};
        a.lse = lse + t0;
        a.row = row + t0;
        by_shape<F>(size, [&](auto shape) {
          typedef decltype(shape) S;
          a.tiles_m = tiles_of(vs, S::BM);
          a.tiles_n = tiles_of(ts, S::BN);
          loss_gradient_kernel<F, T, S>
              <<<mm_grid((uint64_t)a.tiles_m * a.tiles_n, S::kMost), S::kThreads, S::kLds, s>>>(a);
        });
        Product ph{}, pw{};
        ph.pitch = pw.pitch = l.k;
        by_shape<F>(l.spread.size, [&](auto shape) {
          typedef decltype(shape) S;
          if (dh) {
            ph.a = {a.g, l.piece, ts, a.g_plane};
            ph.b = a.w;
            ph.b.rows = n;
            ph.k = vs;
            ph.planes_b = 1;
            ph.rows = ts;
            ph.out = sums_h + t0 * l.k;
            ph.split = rows * l.k;
            ph.add = v0 > 0;
            ph.final = {(F*)dh + t0 * n, n, factor, nullptr, row + t0};
            cut<S>(ph, l.spread.splits_h);
            if (l.sum_h) ph.final.out = nullptr;
          }
          if (dtable) {
            pw.a = {a.g, l.piece, l.piece, a.g_plane};
            pw.b = {(const T*)(w + l.weighed) + t0 * l.k, l.k, n, rows * l.k};
            pw.k = ts;
            pw.planes_b = l.weighed_planes;
            pw.rows = vs;
            pw.out = sums_w;
            pw.split = l.piece * l.k;
            pw.add = t0 > 0;
            pw.final = final_w;
            cut<S>(pw, l.spread.splits_w);
            if (l.sum_w) pw.final.out = nullptr;
          }
          const uint64_t tiles = (uint64_t)ph.tiles_m * ph.tiles_n * ph.splits +
                                 (uint64_t)pw.tiles_m * pw.tiles_n * pw.splits;
          loss_product_kernel<F, T, S>
              <<<mm_grid(tiles, S::kMost), S::kThreads, S::kLds, s>>>(ph, pw);
        });
      }
      if (dtable && l.sum_w)
        finish<F>(sums_w, vs, l.k, l.piece * l.k, l.spread.splits_w, final_w, s);
    }
    if (dh && l.sum_h) finish<F>(sums_h, rows, l.k, rows * l.k, l.spread.splits_h, final_h, s);
  });
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}
