// attn_kernels.h -- attention over packed sequences, forward and backward, on 32x32
// MFMA tiles.
//
//   S = scale Q K^T + bias, P = softmax(S), O = P V
//   D = rowsum(dO O), dP = dO V^T, dS = P (dP - D)
//   dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO, dbias = sums of dS by bucket
//
// Every product is laid out so that one lane holds one row of queries (forward, dQ)
// or one key (dK, dV) and its registers run along the axis that is summed next:
//
//   S^T = K Q^T puts query lane % 32 in a lane, and keys 8 g + 4 (lane / 32) + t in
//   register 4 g + t.  The row's maximum and sum are then sums over registers and one
//   exchange between the wave's halves, the rescale of O^T = V^T P^T is by a lane's own
//   factor, and the registers 8 s .. 8 s + 7 already are the B operand of the next
//   product's 16-key step s, with the keys in the order {16 s + 4 h + 0..3,
//   16 s + 8 + 4 h + 0..3}.  The order of a sum's terms is free as long as both operands
//   agree, so the A operand (V^T, K^T) is read from LDS in that order: two transposing
//   8-byte reads for 16-bit values, eight 4-byte reads for 32-bit ones.  Probabilities
//   never pass through LDS.
//
// The tiles are loaded one ahead, straight into LDS where the rows may be moved in 16-byte
// pieces.  An LDS row's pieces are permuted by its number (piece_of) so that both ways to
// read a tile touch every bank equally.  Rows that a mask leaves out, or past the sequence's
// end, are zeros there: what they hold never meets a product.
//
// P and dS are rounded to the inputs' type for the second products, as those run on the
// 16-bit matrix units; S, dP, the statistics (of P before it is rounded; only the output's
// divisor is of P as the product takes it) and every accumulator are fp32.  bfloat16
// keeps fp32's range.  binary16 does not, so there the values are scaled by powers of two
// that the end takes out exactly: P by 2^11 at the running maximum (forward) or by 2^14
// (dV, where P <= 1), and dS by what brings its largest magnitude to 2^13 .. 2^14.
#pragma once

#include <type_traits>

#include "attn.h"
#include "once_per_device.h"

namespace sieve {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T>
struct Vec8 {
  typedef T type __attribute__((ext_vector_type(8)));
};
template <typename T>
using vec8 = typename Vec8<T>::type;

__device__ __forceinline__ f32x16 mma(vec8<f16> a, vec8<f16> b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(vec8<bf16> a, vec8<bf16> b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// 16 terms in fp32: step j multiplies element j of both halves' operands
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// An LDS tile has rows of kPitch values: DP, or the next power of two.  Piece c (16 bytes) of
// row r lies at piece c ^ piece_of(r) of the row.  64 banks of 4 bytes hold 16 pieces: a row (or
// two, or four of the shorter ones).  Along the head (32 rows, one piece of each) and across the
// rows (4 rows by 2 or 4 neighbouring pieces, twice) every 16 pieces then fall on 16 different
// places.
template <int DP>
constexpr int kPitch = DP == 96 ? 128 : DP;

template <typename T, int DP>
__device__ __forceinline__ int piece_of(int row) {
  constexpr int kPieces = kPitch<DP> * (int)sizeof(T) / 16;
  if constexpr (kPieces >= 16) return (row & 3) << 2 | (row >> 2 & 3);
  else if constexpr (kPieces == 8) return (row & 2) << 1 | (row >> 2 & 3);
  else return row >> 2 & 3;
}

// LDS is addressed by its own 32-bit byte addresses: a lane's place in a tile is worked out
// once, and what a read adds to it is an exclusive or with a constant and a constant offset
// (tiles start at multiples of their rows' bytes: the kernels have no LDS but the dynamic
// part, which starts at 0).
typedef uint32_t lds_addr;
template <typename V>
__device__ __forceinline__ V lds_read(lds_addr at) {
  return *(const __attribute__((address_space(3))) V*)(uintptr_t)at;
}
template <typename V>
__device__ __forceinline__ void lds_write(lds_addr at, V v) {
  *(__attribute__((address_space(3))) V*)(uintptr_t)at = v;
}
__device__ __forceinline__ lds_addr lds_of(const void* p) {
  return (lds_addr)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// A lane's place for frag_along and frag_across, from the start of a tile.
template <typename T, int DP>
__device__ __forceinline__ lds_addr lane_along(int lane) {
  const int row = lane & 31, h = lane >> 5;
  return row * kPitch<DP> * (int)sizeof(T) +
         ((sizeof(T) == 2 ? h : 2 * h) ^ piece_of<T, DP>(row)) * 16;
}
template <typename T, int DP>
__device__ __forceinline__ lds_addr lane_across(int lane) {
  const int h = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int i = lane & 15, row = 4 * h + (i >> 2);
    const int piece = (lane >> 3 & 2) + (i >> 1 & 1);
    return row * kPitch<DP> * 2 + (piece ^ piece_of<T, DP>(row)) * 16 + (i & 1) * 8;
  } else {
    // rows 4 h + 0..3: the row's number within 4 changes piece_of by a constant
    return 4 * h * kPitch<DP> * 4 + ((lane & 31) / 4 ^ piece_of<T, DP>(4 * h)) * 16 +
           (lane & 3) * 4;
  }
}

// Values 16 c + 8 h .. + 7 of the rows row0 + lane % 32 (row0 a multiple of 32): the operand
// whose summed axis is the head's.  at: the tile's start plus lane_along.
template <typename T, int DP>
__device__ __forceinline__ vec8<T> frag_along(lds_addr at, int row0, int c) {
  const int add = row0 * kPitch<DP> * (int)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    return __builtin_bit_cast(vec8<T>, lds_read<enc_u32x4>((at ^ (32 * c)) + add));
  } else {
    const f32x4 p = lds_read<f32x4>((at ^ (64 * c)) + add);
    const f32x4 q = lds_read<f32x4>((at ^ (64 * c) ^ 16) + add);
    return __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// Operands that a wave keeps in LDS for itself, in the lanes' order: chunk c at
// at + c * kFragBytes, at being the wave's place plus 16 bytes a lane.
template <typename T>
constexpr int kFragBytes = 64 * 8 * (int)sizeof(T);
template <typename T>
__device__ __forceinline__ vec8<T> frag_kept(lds_addr at, int c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_bit_cast(vec8<T>, lds_read<enc_u32x4>(at + c * kFragBytes<T>));
  } else {
    const f32x4 p = lds_read<f32x4>(at + c * kFragBytes<T>);
    const f32x4 q = lds_read<f32x4>(at + c * kFragBytes<T> + 1024);
    return __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}
template <typename T>
__device__ __forceinline__ void keep_frag(lds_addr at, int c, vec8<T> v) {
  if constexpr (sizeof(T) == 2) {
    lds_write(at + c * kFragBytes<T>, __builtin_bit_cast(enc_u32x4, v));
  } else {
    lds_write(at + c * kFragBytes<T>, __builtin_shufflevector(v, v, 0, 1, 2, 3));
    lds_write(at + c * kFragBytes<T> + 1024, __builtin_shufflevector(v, v, 4, 5, 6, 7));
  }
}

// Value col + lane % 32 of the rows row0 + {4 h + 0..3, 8 + 4 h + 0..3} (row0 a multiple of
// 16, col of 32): the operand whose summed axis is the tile's rows.  The transposing read
// gives lane i of each 16 the i-th column of the 4 rows that the 16 lanes' addresses cover.
// at: the tile's start plus lane_across.
template <typename T, int DP>
__device__ __forceinline__ vec8<T> frag_across(lds_addr at, int row0, int col) {
  constexpr int kRow = kPitch<DP> * (int)sizeof(T);
  const int x = col * (int)sizeof(T), add = row0 * kRow;
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    union {
      s16x4 half[2];
      vec8<T> all;
    } u;
    // 8 rows on, piece_of differs in bit 1
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)((at ^ x) + add));
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4*)(uintptr_t)((at ^ x ^ 32) + add + 8 * kRow));
    return u.all;
  } else {
    vec8<T> r;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int row = (j & 3) + (j & 4) * 2;
      r[j] = lds_read<float>((at ^ x ^ (piece_of<T, DP>(row) * 16)) + add + row * kRow);
    }
    return r;
  }
}

// Registers 8 s .. 8 s + 7 as an operand, rounded to nearest.
template <typename T>
__device__ __forceinline__ vec8<T> frag_of(const f32x16& x, int s) {
  const f32x8 v = s == 0 ? __builtin_shufflevector(x, x, 0, 1, 2, 3, 4, 5, 6, 7)
                         : __builtin_shufflevector(x, x, 8, 9, 10, 11, 12, 13, 14, 15);
  return __builtin_convertvector(v, vec8<T>);
}

// Query of packed row r: r / G for r < 2^31, by the multiplier ceil(2^(31 + s) / G) with
// 2^(s-1) < G <= 2^s (its excess over the quotient is below 2^s, so the error stays below 1/G).
__device__ __forceinline__ int query_of(const AttnArgs& a, int r) {
  return (int)(__umulhi((uint32_t)r << 1, a.g_mul) >> a.g_shift);
}

// The value of the lane 32 away.
__device__ __forceinline__ float other_half(float v) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  // lanes 32..63 of the first and 0..31 of the second change places
  const u32x2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

// The wave's number, known to be the same in all lanes.
__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
}

// Offset of packed row r (query r / G, head r % G of the group).
__device__ __forceinline__ int64_t row_at(const AttnArgs& a, const sieve_heads& x,
                                          const AttnItem& it, int r) {
  const int tok = query_of(a, r);
  return (it.q0 + tok) * x.token_stride +
         (int64_t)(it.kvh * a.G + (r - tok * a.G)) * x.head_stride;
}

// One row's values 16 c + 8 h .. + 7 for all c, from global memory; zeros past the head's
// size, or all zeros where the row is not there.
template <typename T, int DP, bool kVec>
__device__ __forceinline__ void load_frags(const T* p, bool ok, int d, int h,
                                           vec8<T> (&f)[DP / 16]) {
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) {
    const int col = 16 * c + 8 * h;
    EncVec<T, 8> q;
#pragma unroll
    for (int j = 0; j < 8; ++j) q.v[j] = (T)0.f;
    if (ok && col < d) {
      if constexpr (kVec && sizeof(T) == 2) {
        q = enc_load<T, 8>(p + col);
      } else if constexpr (kVec) {  // d is a multiple of 4
        const EncVec<T, 4> a = enc_load<T, 4>(p + col);
#pragma unroll
        for (int j = 0; j < 4; ++j) q.v[j] = a.v[j];
        if (col + 4 < d) {
          const EncVec<T, 4> b = enc_load<T, 4>(p + col + 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) q.v[4 + j] = b.v[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j < d) q.v[j] = p[col + j];
      }
    }
    f[c] = __builtin_bit_cast(vec8<T>, q);
  }
}

// Loads of 16 bytes at a 32-bit offset from a base that the whole wave shares; kNowhere loads
// zeros.  A row that is not there costs a select instead of a branch.
constexpr uint32_t kNowhere = 0x80000000u;
struct Buffer {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ explicit Buffer(const void* base)
      : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)kNowhere,
                                               0x00027000)) {}
  __device__ __forceinline__ enc_u32x4 load(uint32_t offset) const {
    return __builtin_bit_cast(enc_u32x4,
                              __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)offset, 0, 0));
  }
  // into LDS, 16 bytes a lane from `to`, which the wave shares
  __device__ __forceinline__ void load_lds(uint32_t offset, void* to) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void*)to, 16, (int)offset, 0, 0, 0);
  }
};

// Waits for the wave's own loads (gfx9 encoding: vmcnt 0, the other counts not waited for).
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);
  asm volatile("" ::: "memory");
}

// A tile of ROWS rows on its way from global memory into LDS, a 16-byte piece a thread at a
// time in the order of their places.  Whether a row counts (a mask, a row without keys) is
// itself loaded: the rows are loaded without waiting for it, and cleared when both are there.
// kVec: the rows may be moved in 16-byte pieces and a tile spans less than 2^31 bytes.
// kDirect: the loads write LDS themselves (the buffer they go to is not being read).
template <typename T, int DP, int ROWS, bool kVec, bool kDirect>
struct Stage {
  static_assert(kVec || !kDirect);
  static constexpr int kE = 16 / sizeof(T);           // values of a 16-byte piece
  static constexpr int kPieces = kPitch<DP> / kE;     // pieces of a row
  static constexpr int kAll = ROWS * kPieces;
  static constexpr int kN = (kAll + kAttnThreads - 1) / kAttnThreads;
  static_assert(kAll % 64 == 0);
  static constexpr bool kDirectLoads = kDirect;
  enc_u32x4 r[kDirect ? 1 : kN];

  // row and first value of this thread's piece i
  static __device__ __forceinline__ int row(int i) {
    return (threadIdx.x + i * kAttnThreads) / kPieces;
  }
  static __device__ __forceinline__ int col(int i) {
    return ((threadIdx.x + i * kAttnThreads) % kPieces ^ piece_of<T, DP>(row(i))) * kE;
  }
  static __device__ __forceinline__ bool mine(int i) {
    return kAll % kAttnThreads == 0 || threadIdx.x + i * kAttnThreads < kAll;
  }
  // Offsets of the pieces from a tile's first row, worked out once: at(row, col) in values,
  // kNowhere past the head's size.
  typedef std::conditional_t<kVec, uint32_t, int64_t> Off;
  Off off[kN];
  template <typename F>
  __device__ __forceinline__ void place(F at, int d) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      if constexpr (kVec)
        off[i] = col(i) < d && mine(i) ? (uint32_t)at(row(i), col(i)) * (uint32_t)sizeof(T)
                                       : kNowhere;
      else
        off[i] = at(row(i), col(i));
    }
  }
  // rows: how many of the tile's there are; s: the tile's place in LDS
  __device__ __forceinline__ void load(const T* base, int rows, int d, T* s) {
    const Buffer from(base);
    if constexpr (kVec) {
      if (rows >= ROWS) {
#pragma unroll
        for (int i = 0; i < kN; ++i) move(from, off[i], i, s);
      } else {
#pragma unroll
        for (int i = 0; i < kN; ++i) move(from, row(i) < rows ? off[i] : kNowhere, i, s);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        EncVec<T, kE> q;
#pragma unroll
        for (int j = 0; j < kE; ++j)
          q.v[j] = mine(i) && row(i) < rows && col(i) + j < d ? base[off[i] + j] : (T)0.f;
        r[i] = __builtin_bit_cast(enc_u32x4, q);
      }
    }
  }
  __device__ __forceinline__ void move(const Buffer& from, uint32_t offset, int i, T* s) {
    if constexpr (kDirect) {
      if (mine(i)) from.load_lds(offset, s + (i * kAttnThreads + wave_id() * 64) * kE);
    } else {
      r[i] = from.load(offset);
    }
  }
  // the pieces are in LDS after this and the next barrier; keep(i): whether piece i counts
  template <typename F>
  __device__ __forceinline__ void store(T* s, bool check, F keep) {
    if constexpr (kDirect) {
      if (check) {
#pragma unroll
        for (int i = 0; i < kN; ++i)
          if (mine(i) && !keep(i))
            *(enc_u32x4*)(s + (threadIdx.x + i * kAttnThreads) * kE) = enc_u32x4{0, 0, 0, 0};
      }
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (mine(i))
          *(enc_u32x4*)(s + (threadIdx.x + i * kAttnThreads) * kE) =
              check && !keep(i) ? enc_u32x4{0, 0, 0, 0} : r[i];
    }
  }
};

// The keys and values of a tile, and what the mask says of their rows.
template <typename T, int DP, int KEYS, bool kVec, bool kDirect>
struct KeyStage {
  using Tile = Stage<T, DP, KEYS, kVec, kDirect>;
  Tile k, v;
  uint8_t keep[Tile::kN];

  __device__ __forceinline__ void place(const AttnArgs& a) {
    const int64_t ks = a.k.token_stride, vs = a.v.token_stride;
    k.place([&](int row, int col) { return row * ks + col; }, a.d);
    v.place([&](int row, int col) { return row * vs + col; }, a.d);
  }
  // k0, v0: the sequence's first row; keys base .. hi - 1 at most
  __device__ __forceinline__ void load(const AttnArgs& a, const uint8_t* mask, const T* k0,
                                       const T* v0, int base, int hi, T* s_k, T* s_v) {
    k.load(k0 + base * a.k.token_stride, hi - base, a.d, s_k);
    v.load(v0 + base * a.v.token_stride, hi - base, a.d, s_v);
    if (mask) {
#pragma unroll
      for (int i = 0; i < Tile::kN; ++i) {
        const int key = base + Tile::row(i);
        keep[i] = key < hi ? mask[key] : 0;
      }
    }
  }
  __device__ __forceinline__ void store(const uint8_t* mask, T* s_k, T* s_v) {
    if (kDirect) wait_loads();
    k.store(s_k, mask != nullptr, [&](int i) { return keep[i] != 0; });
    v.store(s_v, mask != nullptr, [&](int i) { return keep[i] != 0; });
  }
};

// Accumulators X^T (rows: the head's values 32 b + 8 g + 4 h + t in register 4 g + t,
// column: the lane's row) times f, to a row in global memory.
template <typename T, int DP, bool kVec>
__device__ __forceinline__ void store_row(T* p, const f32x16 (&x)[DP / 32], float f, int d,
                                          int h) {
#pragma unroll
  for (int b = 0; b < DP / 32; ++b) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * b + 8 * g + 4 * h;
      typedef T vec4 __attribute__((ext_vector_type(4)));
      const f32x4 v = {x[b][4 * g] * f, x[b][4 * g + 1] * f, x[b][4 * g + 2] * f,
                       x[b][4 * g + 3] * f};
      const vec4 q = __builtin_convertvector(v, vec4);
      if constexpr (kVec) {  // d is a multiple of 4
        if (col < d) *(vec4*)(p + col) = q;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < d) p[col + j] = q[j];
      }
    }
  }
}

// A bias in units of log2, held to +-2^20: past that fp32 keeps nothing of the score it is added
// to, the backward pass could not tell a row's probabilities from its lse, and the lowest values
// of fp32 and bfloat16 would become -infinity.  -infinity itself forbids; NaN stays.
__device__ __forceinline__ float held_bias(float b) {
  constexpr float kMost = 0x1p20f;
  if (b < -kMost && b > -INFINITY) b = -kMost;
  if (b > kMost && b < INFINITY) b = kMost;
  return b * kLog2e;
}

// The group's bias tables into LDS, times log2(e): s[g * span + entry].  The first entries'
// buckets and values are loaded side by side; the values change places within the wave where
// there are at most 64 of them.
template <typename T>
__device__ __forceinline__ void load_bias(const AttnArgs& a, int kvh, float* s) {
  const T* bias = (const T*)a.bias + kvh * a.G;
  if (a.nb <= 64) {
    const int lane = threadIdx.x & 63;
    for (int g = 0; g < a.G; ++g) {
      const float mine = lane < a.nb ? held_bias((float)bias[(int64_t)lane * a.heads + g]) : 0.f;
      for (int i = threadIdx.x; i - lane < a.span; i += kAttnThreads) {
        const int bucket = i < a.span ? a.bucket_of[i] : 0;
        const float v = __shfl(mine, bucket);
        if (i < a.span) s[g * a.span + i] = v;
      }
    }
    return;
  }
  for (int g = 0; g < a.G; ++g)
    for (int i = threadIdx.x; i < a.span; i += kAttnThreads)
      s[g * a.span + i] = held_bias((float)bias[(int64_t)a.bucket_of[i] * a.heads + g]);
}

// Not 0: the key is in the item's range and not masked.  Loaded a tile ahead.
__device__ __forceinline__ uint8_t key_ok(const uint8_t* mask, int key, int hi) {
  if (key >= hi) return 0;
  return mask ? mask[key] : 1;
}

// Bits 0..31: key base + bit is not after position pos.
__device__ __forceinline__ uint32_t upto(int pos, int base) {
  const int lim = pos - base;
  return lim >= 31 ? ~0u : lim < 0 ? 0u : (2u << lim) - 1;
}

// Products of 32 keys (base ..) with the lane's row to scores: s * scale2 + bias, in units of
// log2, and -infinity where bits (of the keys) has a 0.  Without a bias the products stay as
// they are.  lo, hi: bias past the distance; dp: set to 0 in the same places.
template <bool kBias>
__device__ __forceinline__ void finish_scores(f32x16& s, float scale2, const float* table,
                                              int distance, int pos, int pos_min, int pos_max,
                                              float lo, float hi, int base, int h, uint32_t bits,
                                              f32x16* dp = nullptr) {
  if constexpr (kBias) {
    if (base - pos_max >= distance || base + 31 - pos_min <= -distance) {
      const float far = base > pos_min ? hi : lo;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = s[r] * scale2 + far;
    } else {
      const float* t = table + (base + 4 * h - pos + distance + kAttnPad);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = s[r] * scale2 + t[8 * (r >> 2) + (r & 3)];
    }
  }
  if (!__all(bits == ~0u)) {
    const uint32_t mine = bits >> (4 * h);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const bool seen = mine >> (8 * (r >> 2) + (r & 3)) & 1;
      s[r] = seen ? s[r] : -INFINITY;
      if (dp) (*dp)[r] = seen ? (*dp)[r] : 0.f;  // P = 0 there, but dP need not be a number
    }
  }
}

// What a lane knows about its row.
struct LaneRow {
  int r, tok, g, pos;  // row, query, head in the group, position
  int pos_min, pos_max;  // over the wave's rows
  bool live;
};
__device__ __forceinline__ LaneRow lane_row(const AttnArgs& a, const AttnItem& it, int first,
                                            int lane) {
  LaneRow x;
  const int G = a.G;
  const int rows = it.nq * G;
  x.r = first + (lane & 31);
  x.live = x.r < rows;
  const int r = x.live ? x.r : (rows > 0 ? rows - 1 : 0);
  x.tok = query_of(a, r);
  x.g = r - x.tok * G;
  const int shift = it.nk - it.nq;
  x.pos = x.tok + shift;
  const int last = first + 31 < rows ? first + 31 : rows - 1;
  const int head = first < rows ? first : rows - 1;
  x.pos_min = query_of(a, head) + shift;
  x.pos_max = query_of(a, last) + shift;
  return x;
}

// The running maximum may lag by kLag powers of two before the sums are brought to a new one,
// and P is 2^kShift at it.  For binary16, 2^(kLag + kShift) has to stay below 65504 and what
// 2^kShift pushes below 2^-14 loses bits.  2 x 8,192 tokens of 16 heads of 128, bf16: 1,054 us,
// without a lag 1,100; 4 x 8,192 of 12 heads of 64: 926, 962.
template <typename T>
constexpr float kLag = __is_same(T, f16) ? 4.f : 8.f;
template <typename T>
constexpr float kShift = __is_same(T, f16) ? 11.f : 0.f;

// x plus the sum of an operand's eight values: of the rounded probabilities, which are what
// the second product adds up and so what its result is divided by, two to an instruction.
// lse is of the probabilities before they are rounded, summed in fp32 beside them.
__device__ __forceinline__ float add_up(vec8<f16> p, float x) {
  typedef f16 pair __attribute__((ext_vector_type(2)));
  const pair one = {(f16)1.f, (f16)1.f};
  x = __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 0, 1), one, x, false);
  x = __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 2, 3), one, x, false);
  x = __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 4, 5), one, x, false);
  return __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 6, 7), one, x, false);
}
__device__ __forceinline__ float add_up(vec8<bf16> p, float x) {
  typedef bf16 pair __attribute__((ext_vector_type(2)));
  const pair one = {(bf16)1.f, (bf16)1.f};
  x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 0, 1), one, x, false);
  x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 2, 3), one, x, false);
  x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 4, 5), one, x, false);
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 6, 7), one, x, false);
}
__device__ __forceinline__ float add_up(f32x8 p, float x) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x += p[j];
  return x;
}

// Whether the 32 rows from row0 of a tile hold an infinity or NaN in the wave's columns.
// (A bfloat16 sum may also overflow: the answer is then the careful path, which is right too.)
template <typename T, int DP>
__device__ __forceinline__ bool odd_values(lds_addr at, int row0) {
  float x = 0.f;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int e = 0; e < DP / 32; ++e)
      x = add_up(frag_across<T, DP>(at, row0 + 16 * c, 32 * e), x);
  return __any(!(fabsf(x) < INFINITY));
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// One row again, without products of keys that it does not see: where a block that causal
// rows see in part holds infinities or NaN, 0 times such a value would reach the rows before
// it.  A wave a row, 64 keys at a time, a key a lane for the scores and two values a lane for
// the sums.  Rare, and slow next to the products it replaces.
//   kGrad = false: acc += P v relative to 2^m, with the sum l; true: acc += dS k, with m the
//   row's lse in units of log2 and l its D.
template <typename T, bool kBias, bool kGrad>
__device__ void careful_row(const AttnArgs& a, const AttnItem& it, const float* bias, int r,
                            int lane, float (&acc)[2], float& m, float& l) {
  const int tok = query_of(a, r), pos = tok + it.nk - it.nq, d = a.d;
  const float* table = kBias ? bias + (r - tok * a.G) * a.span : nullptr;
  const T* q = (const T*)a.q.data + row_at(a, a.q, it, r);
  const T* dout = kGrad ? (const T*)a.dout.data + row_at(a, a.dout, it, r) : nullptr;
  const T* k0 = (const T*)a.k.data + it.k0 * a.k.token_stride + it.kvh * a.k.head_stride;
  const T* v0 = (const T*)a.v.data + it.k0 * a.v.token_stride + it.kvh * a.v.head_stride;
  const float scale2 = a.scale * kLog2e;
  acc[0] = acc[1] = 0.f;
  if (!kGrad) {
    m = -INFINITY;
    l = 0.f;
  }
  const int end = a.causal && pos + 1 < it.hi ? pos + 1 : it.hi;
  for (int base = it.lo; base < end; base += 64) {
    const int key = base + lane;
    const bool seen = key < end && (!a.key_mask || a.key_mask[it.k0 + key] != 0);
    float s = -INFINITY, dp = 0.f;
    if (seen) {
      const T* k = k0 + key * a.k.token_stride;
      s = 0.f;
      for (int c = 0; c < d; ++c) s += (float)q[c] * (float)k[c];
      s *= scale2;
      if (kBias) {
        int rel = key - pos;
        rel = rel < -a.distance ? -a.distance : rel > a.distance ? a.distance : rel;
        s += table[rel + a.distance + kAttnPad];
      }
      if (kGrad) {
        const T* v = v0 + key * a.v.token_stride;
        for (int c = 0; c < d; ++c) dp += (float)dout[c] * (float)v[c];
      }
    }
    float x;  // what the key's row is multiplied with
    if (kGrad) {
      x = seen ? __builtin_amdgcn_exp2f(s - m) * (dp - l) : 0.f;
    } else {
      const float next = fmaxf(m, wave_max(s)), at = next == -INFINITY ? 0.f : next;
      const float f = __builtin_amdgcn_exp2f(m - at);
      x = seen ? __builtin_amdgcn_exp2f(s - at) : 0.f;
      l = l * f + wave_add(x);
      acc[0] *= f;
      acc[1] *= f;
      m = next;
    }
    const uint64_t these = __ballot(seen);
    for (int j = 0; j < 64; ++j) {
      if (!(these >> j & 1)) continue;
      const float xj = __shfl(x, j);
      const T* row = kGrad ? k0 + (int64_t)(base + j) * a.k.token_stride
                           : v0 + (int64_t)(base + j) * a.v.token_stride;
      if (lane < d) acc[0] += xj * (float)row[lane];
      if (lane + 64 < d) acc[1] += xj * (float)row[lane + 64];
    }
  }
}

// The kernel's arguments, read again from where the launch put them (its one parameter is the
// first thing there).  A rare path that takes them from here does not keep the ones that only it
// needs in scalar registers over the loop before it.
__device__ __forceinline__ AttnArgs args_again() {
  typedef const __attribute__((address_space(4))) uint64_t* Words;
  static_assert(sizeof(AttnArgs) % 8 == 0 && std::is_trivially_copyable<AttnArgs>::value);
  Words from = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(from));
  uint64_t words[sizeof(AttnArgs) / 8];
#pragma unroll
  for (size_t i = 0; i < sizeof(AttnArgs) / 8; ++i) words[i] = from[i];
  AttnArgs a;
  __builtin_memcpy(&a, words, sizeof(a));
  return a;
}

// One key's gradients again, without products of rows that do not see it: the mirror image of
// the above for dK and dV, where a block that is causal in part holds infinities or NaN in q or
// dout.  A wave a key, 64 rows at a time, a row a lane for P and dS and two values a lane for
// the sums: dk += dS q, dv += P dout.
template <typename T, bool kBias>
__device__ void careful_key(const AttnArgs& a, const AttnItem& it, const float* bias, int key,
                            int lane, float (&dk)[2], float (&dv)[2]) {
  const int d = a.d, shift = it.nk - it.nq;
  const T* k = (const T*)a.k.data + (it.k0 + key) * a.k.token_stride + it.kvh * a.k.head_stride;
  const T* v = (const T*)a.v.data + (it.k0 + key) * a.v.token_stride + it.kvh * a.v.head_stride;
  const float scale2 = a.scale * kLog2e;
  dk[0] = dk[1] = dv[0] = dv[1] = 0.f;
  for (int base = it.lo; base < it.hi; base += 64) {
    const int r = base + lane;
    float p = 0.f, ds = 0.f;
    bool sees = false;
    if (r < it.hi) {
      const int tok = query_of(a, r), pos = tok + shift, g = r - tok * a.G;
      const int64_t at = (it.q0 + tok) * a.heads + it.kvh * a.G + g;
      const float lse = a.lse[at];
      sees = key <= pos && lse != -INFINITY;
      if (sees) {
        const T* q = (const T*)a.q.data + row_at(a, a.q, it, r);
        const T* dout = (const T*)a.dout.data + row_at(a, a.dout, it, r);
        float s = 0.f, dp = 0.f;
        for (int c = 0; c < d; ++c) {
          s += (float)q[c] * (float)k[c];
          dp += (float)dout[c] * (float)v[c];
        }
        s *= scale2;
        if (kBias) {
          int rel = key - pos;
          rel = rel < -a.distance ? -a.distance : rel > a.distance ? a.distance : rel;
          s += bias[g * a.span + rel + a.distance + kAttnPad];
        }
        p = __builtin_amdgcn_exp2f(s - lse * kLog2e);
        ds = p * (dp - a.dsum[at]);
      }
    }
    const uint64_t these = __ballot(sees);
    for (int j = 0; j < 64; ++j) {
      if (!(these >> j & 1)) continue;
      const float pj = __shfl(p, j), dsj = __shfl(ds, j);
      const T* q = (const T*)a.q.data + row_at(a, a.q, it, base + j);
      const T* dout = (const T*)a.dout.data + row_at(a, a.dout, it, base + j);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < d) {
          dk[e] += dsj * (float)q[lane + 64 * e];
          dv[e] += pj * (float)dout[lane + 64 * e];
        }
    }
  }
}

// Work-groups a CU that a kernel's registers are to leave room for.
template <typename T, int DP>
constexpr int kGroupsPerCu = sizeof(T) * DP > 256 ? 1 : 2;

// ---- forward ----------------------------------------------------------------------------
// WK = 1: a wave takes 32 of the tile's 128 rows and all keys.  WK = 4: the tile is 32 rows,
// each wave takes every fourth block of 32 keys, and LDS joins the four at the end: for
// few rows, where the keys' and values' bytes bound the time.  Long sequences: matrix and
// vector issue (matrix units 36-38% busy); 12,007 causal tokens, 16 heads over 4 of 128, bf16,
// 718 us, 823 TFLOP/s (of it 28 us for the sum that lse is made from).  Few rows: memory; one
// query over 32 documents of 1,000..30,000 224 us with the join, 4.9 TB/s.  Tiles of 64 keys:
// with 32 the 12,007 tokens took 755 us against 670, 4 x 8,192 of 12 heads of 64 977 against 926
// (before that sum).

template <typename T, int DP, int WK>
struct FwdShape {
  static constexpr int kBlocks = WK == 1 && sizeof(T) == 2 ? 2 : 1;  // 32-key blocks of a wave
  static constexpr int kTile = 32 * kBlocks * WK;                    // keys of a tile
  static constexpr int kTileBytes = kTile * kPitch<DP> * (int)sizeof(T);
  static constexpr int kBufs = 4 * kTileBytes <= 128 * 1024 ? 2 : 1;
  static constexpr int kStageBytes = 2 * kBufs * kTileBytes;
  static constexpr int kJoinBytes =
      WK == 1 ? 0 : (WK * 32 * (DP + 4) + kAttnStats * WK * 32 + WK) * 4;
  static constexpr int kBytes = kStageBytes > kJoinBytes ? kStageBytes : kJoinBytes;
  static constexpr int kRows = WK == 1 ? kAttnRows : kAttnFewRows;
};

template <typename T, int DP, int WK, bool kBias, bool kVec>
__global__ __launch_bounds__(kAttnThreads, (kGroupsPerCu<T, DP>)) void attn_forward_kernel(
    AttnArgs a) {
  using Shape = FwdShape<T, DP, WK>;
  constexpr int kBlocks = Shape::kBlocks, kTile = Shape::kTile;
  constexpr int kTileN = kTile * kPitch<DP>;
  constexpr bool kTwoSums = sizeof(T) == 2;
  extern __shared__ __align__(16) uint8_t smem[];
  T* s_k = (T*)smem;
  T* s_v = s_k + Shape::kBufs * kTileN;
  float* s_bias = (float*)(smem + Shape::kBytes);
  const AttnItem it = a.items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5;
  const int G = a.G, d = a.d;
  const LaneRow me = lane_row(a, it, it.row + (WK == 1 ? wave * 32 : 0), lane);
  const float scale2 = a.scale * kLog2e;
  const bool wave_live = WK == 4 || it.row + wave * 32 < it.nq * G;

  const T* k0 = (const T*)a.k.data + it.k0 * a.k.token_stride + it.kvh * a.k.head_stride;
  const T* v0 = (const T*)a.v.data + it.k0 * a.v.token_stride + it.kvh * a.v.head_stride;
  const uint8_t* mask = a.key_mask ? a.key_mask + it.k0 : nullptr;
  KeyStage<T, DP, kTile, kVec, kVec && Shape::kBufs == 2> stage;
  stage.place(a);
  uint8_t ok[kBlocks];
  auto fetch = [&](int base, int b) {
    stage.load(a, mask, k0, v0, base, it.hi, s_k + b * kTileN, s_v + b * kTileN);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
      if (mask || base + kTile > it.hi)
        ok[i] = key_ok(mask, base + 32 * ((WK == 1 ? 0 : wave) + i) + (lane & 31), it.hi);
  };
  if (it.lo < it.hi) fetch(it.lo, 0);

  vec8<T> q[DP / 16];
  {
    const T* p = (const T*)a.q.data + (me.live ? row_at(a, a.q, it, me.r) : 0);
    load_frags<T, DP, kVec>(p, me.live, d, h, q);
  }
  float lo = 0.f, hi = 0.f;
  const float* table = nullptr;
  if constexpr (kBias) {
    load_bias<T>(a, it.kvh, s_bias);
    __syncthreads();
    table = s_bias + me.g * a.span;
    lo = table[0];
    hi = table[a.span - 1];
  }
  f32x16 o[DP / 32];
#pragma unroll
  for (int b = 0; b < DP / 32; ++b) o[b] = f32x16{};
  float m = -INFINITY, l = 0.f, full = 0.f;  // full: l of the probabilities as they were
  bool odd = false;  // the wave's rows have to be done again (careful_row)
  const int skip = WK == 1 ? 0 : wave * 32 * kPitch<DP>;  // the wave's keys in a tile
  const lds_addr k_al = lds_of(s_k + skip) + lane_along<T, DP>(lane);
  const lds_addr v_ac = lds_of(s_v + skip) + lane_across<T, DP>(lane);

  int buf = 0;
  if (it.lo < it.hi) {
    stage.store(mask, s_k, s_v);
    __syncthreads();
  }
  for (int base = it.lo; base < it.hi; base += kTile) {
    const int first = base + (WK == 1 ? 0 : wave * 32);
    uint32_t bits[kBlocks], any = 0;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      bits[b] = mask || base + kTile > it.hi ? (uint32_t)__ballot(ok[b] != 0) : ~0u;
      if (a.causal) bits[b] &= upto(me.pos, first + 32 * b);
      any |= bits[b];
    }
    const bool more = base + kTile < it.hi;
    if (more) fetch(base + kTile, buf ^ (Shape::kBufs - 1));
    if (wave_live && __any(any != 0)) {
      const lds_addr sk = k_al + buf * kTileN * (int)sizeof(T);
      const lds_addr sv = v_ac + buf * kTileN * (int)sizeof(T);
      f32x16 s[kBlocks];
      // the matrix unit first to the wave that feeds it: 3% at heads of 128 values
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        s[b] = f32x16{};
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
          if (sizeof(T) == 4 && 16 * c >= d) break;  // zeros; 8 slow products each
          s[b] = mma(frag_along<T, DP>(sk, 32 * b, c), q[c], s[b]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        finish_scores<kBias>(s[b], scale2, table, a.distance, me.pos, me.pos_min, me.pos_max, lo,
                             hi, first + 32 * b, h, bits[b]);
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
      }
      top = fmaxf(top, other_half(top));
      if constexpr (!kBias) top *= scale2;
      if (__any(top > m + kLag<T>)) {
        const float next = fmaxf(m, top);
        const float f = __builtin_amdgcn_exp2f(m - (next == -INFINITY ? 0.f : next));
        m = next;
        l *= f;
        full *= f;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[b][r] *= f;
      }
      const float off = (m == -INFINITY ? 0.f : m) - kShift<T>;
      if (a.causal) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
          if (!__all(bits[b] == ~0u)) odd |= odd_values<T, DP>(sv, 32 * b);
      }
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[b][r] = __builtin_amdgcn_exp2f(kBias ? s[b][r] - off : s[b][r] * scale2 - off);
        if constexpr (kTwoSums) {
#pragma unroll
          for (int r = 0; r < 16; ++r) full += s[b][r];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const vec8<T> p = frag_of<T>(s[b], c);
          l = add_up(p, l);
#pragma unroll
          for (int e = 0; e < DP / 32; ++e)
            o[e] = mma(frag_across<T, DP>(sv, 32 * b + 16 * c, 32 * e), p, o[e]);
        }
      }
    }
    if (Shape::kBufs == 1) __syncthreads();
    if (more) {
      buf ^= Shape::kBufs - 1;
      stage.store(mask, s_k + buf * kTileN, s_v + buf * kTileN);
      __syncthreads();
    }
  }
  l += other_half(l);
  full = kTwoSums ? full + other_half(full) : l;
  float at = (m == -INFINITY ? 0.f : m) - kShift<T>;  // the sums are relative to 2^at

  if constexpr (WK == 4) {
    // join the waves: sums relative to the largest maximum
    float* s_o = (float*)smem;
    float* s_ml = s_o + WK * 32 * (DP + 4);
    int* s_odd = (int*)(s_ml + kAttnStats * WK * 32);
    __syncthreads();
    if (lane == 0) s_odd[wave] = odd;
    if (h == 0) {
      float* p = s_ml + (wave * 32 + lane) * kAttnStats;
      p[0] = l == 0.f ? -INFINITY : at;
      p[1] = l;
      p[2] = full;
    }
    __syncthreads();
    odd = s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3];
    float most = -INFINITY, sum = 0.f, full_sum = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) most = fmaxf(most, s_ml[(w * 32 + (lane & 31)) * kAttnStats]);
    if (most == -INFINITY) most = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float* p = s_ml + (w * 32 + (lane & 31)) * kAttnStats;
      const float f = p[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(p[0] - most);
      sum += p[1] * f;
      full_sum += p[2] * f;
    }
    const float f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(at - most);
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = {o[b][4 * g] * f, o[b][4 * g + 1] * f, o[b][4 * g + 2] * f,
                         o[b][4 * g + 3] * f};
        *(f32x4*)(s_o + (wave * 32 + (lane & 31)) * (DP + 4) + 32 * b + 8 * g + 4 * h) = v;
      }
    __syncthreads();
    if (wave && !odd) return;
    l = sum;
    full = full_sum;
    at = most;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v = {};
#pragma unroll
        for (int w = 0; w < WK; ++w)
          v += *(const f32x4*)(s_o + (w * 32 + (lane & 31)) * (DP + 4) + 32 * b + 8 * g + 4 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[b][4 * g + j] = v[j];
      }
  }
  if (__builtin_expect(odd, 0)) {
    const int each = 32 / WK, first = WK == 1 ? wave * 32 : wave * each;
    for (int i = first; i < first + each && it.row + i < it.nq * G; ++i) {
      float acc[2], max_, sum_;
      careful_row<T, kBias, false>(a, it, s_bias, it.row + i, lane, acc, max_, sum_);
      const int64_t slot = (int64_t)it.part * Shape::kRows + i;
      const int r = it.row + i, tok = query_of(a, r);
      const float inv = sum_ == 0.f ? 0.f : 1.f / sum_;
#pragma unroll
      for (int e = 0; e < (DP + 63) / 64; ++e) {
        const int col = lane + 64 * e;
        if (it.part >= 0) {
          if (col < DP) a.part_o[slot * DP + col] = acc[e];
        } else if (col < d) {
          ((T*)a.o.data + row_at(a, a.o, it, r))[col] = (T)(acc[e] * inv);
        }
      }
      if (lane == 0) {
        if (it.part >= 0) {
          a.part_ml[slot * kAttnStats] = max_;
          a.part_ml[slot * kAttnStats + 1] = a.part_ml[slot * kAttnStats + 2] = sum_;
        } else if (a.lse) {
          a.lse[(it.q0 + tok) * a.heads + it.kvh * G + (r - tok * G)] =
              sum_ == 0.f ? -INFINITY : (max_ + __builtin_amdgcn_logf(sum_)) * kLn2;
        }
      }
    }
    return;
  }
  if (it.part >= 0) {
    const int64_t slot = (int64_t)it.part * Shape::kRows + (WK == 1 ? wave * 32 : 0) + (lane & 31);
    float* p = a.part_o + slot * DP;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(p + 32 * b + 8 * g + 4 * h) =
            f32x4{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
    if (h == 0) {
      a.part_ml[slot * kAttnStats] = l == 0.f ? -INFINITY : at;
      a.part_ml[slot * kAttnStats + 1] = l;
      a.part_ml[slot * kAttnStats + 2] = full;
    }
    return;
  }
  if (!me.live) return;
  store_row<T, DP, kVec>((T*)a.o.data + row_at(a, a.o, it, me.r), o,
                   l == 0.f ? 0.f : 1.f / l, d, h);
  if (a.lse && h == 0)
    a.lse[(it.q0 + me.tok) * a.heads + it.kvh * G + me.g] =
        l == 0.f ? -INFINITY : (at + __builtin_amdgcn_logf(full)) * kLn2;
}

// Partial rows of one tile to whole ones: DP / 4 threads a row, kJoinRows rows a work-group.
// Latency: 12 us after the pooled queries above.
template <int DP>
constexpr int kJoinRows = kAttnThreads / (DP / 4);

template <typename T, int DP, int ROWS>
__global__ __launch_bounds__(kAttnThreads) void attn_join_kernel(AttnArgs a) {
  constexpr int kGroups = (ROWS + kJoinRows<DP> - 1) / kJoinRows<DP>;
  const AttnJoin j = a.joins[blockIdx.x / kGroups];
  const int i = blockIdx.x % kGroups * kJoinRows<DP> + threadIdx.x / (DP / 4);
  const int r = j.row + i, c = threadIdx.x % (DP / 4) * 4;
  if (threadIdx.x >= kJoinRows<DP> * (DP / 4) || i >= ROWS || r >= j.n * a.G) return;
  const float* ml = a.part_ml + ((int64_t)j.part0 * ROWS + i) * kAttnStats;
  float most = -INFINITY;
#pragma unroll 4
  for (int p = 0; p < j.parts; ++p) most = fmaxf(most, ml[(int64_t)p * ROWS * kAttnStats]);
  if (most == -INFINITY) most = 0.f;
  const float* o = a.part_o + ((int64_t)j.part0 * ROWS + i) * DP + c;
  float l = 0.f, full = 0.f;
  f32x4 v = {};
#pragma unroll 4
  for (int p = 0; p < j.parts; ++p) {
    const float* at = ml + (int64_t)p * ROWS * kAttnStats;
    // a part without keys has l = 0 and o = 0
    const float f = at[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(at[0] - most);
    l += at[1] * f;
    full += at[2] * f;
    v += *(const f32x4*)(o + (int64_t)p * ROWS * DP) * f;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int tok = query_of(a, r), head = j.kvh * a.G + (r - tok * a.G);
  T* to = (T*)a.o.data + (j.t0 + tok) * a.o.token_stride + head * a.o.head_stride + c;
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (c + t < a.d) to[t] = (T)(v[t] * inv);
  if (a.lse && c == 0)
    a.lse[(j.t0 + tok) * a.heads + head] =
        l == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(full)) * kLn2;
}

// The backward pass's probabilities are at most 1 and are computed times 2^kUp: the exponential
// unit returns 0 for results below the normal range, which this leaves room for.
constexpr float kUp = 24.f, kUpOut = 0x1p-24f;

// 2^(v + kUp) for what a row's statistics leave of a score.  In 16 bits the statistics have kUp in
// them already (kUpIn).  In 32 bits that costs bits: next to 24 the exponent's argument is off by
// up to 2^-20, and a probability by 11 times 2^-24.  There kUp is added only to arguments far below
// 0, which are rounded to more than that, and the others' results are multiplied.  Training step
// of 100 masked documents (8 heads of 40): 417 us, gradients 1.16-1.18 times as far from 64 bits
// as the plain form's; with kUp in the statistics 409 us, 1.52-1.57 times.
template <typename T>
constexpr float kUpIn = sizeof(T) == 2 ? kUp : 0.f;
template <typename T>
__device__ __forceinline__ float exp2_up(float v) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_exp2f(v);
  } else {
    const bool low = v < -64.f;
    return __builtin_amdgcn_exp2f(low ? v + kUp : v) * (low ? 1.f : 1.f / kUpOut);
  }
}

// ---- backward: dQ and the bias table's gradient ------------------------------------------
// A wave takes 32 of the tile's 128 rows and goes through the keys as the forward pass does.
// It writes D for the second kernel.
//
// The bias table's gradient is a sum along diagonals.  Where a block of keys is past the
// distance it all falls into one bucket, and the lane adds it up in a register.  Nearer, the
// wave writes its 32x32 block of dS to LDS, 16 rows at a time, with zeros beside every row, so
// that a lane can read down a whole diagonal without a test (row i's value at relative
// position p + i lies at a constant step from row i - 1's), and adds the result to its own
// sums by position.  No atomics: the order of additions is the program's.
//
// Issue bounds it.  Two causal documents of 5,000..6,100 (16 heads over 4 of 128, bf16) 459 us;
// 256 documents of 16..512 (12 heads of 64, f16) with a bias's gradient 371.  That gradient adds
// 70 to 110 us to a backward pass of 552 to 560.
//
// dS is rounded to the inputs' type for the product and D comes from the rounded output: dQ and
// dK in 16 bits are up to 1.8 times as far from exact as one rounding of the result.

// With a bias the tile is 32 keys, so that two work-groups' LDS fits a CU beside the sums: the
// 256 documents' backward pass takes 630 us, with 64 keys 749.  Without one 64 keys are faster
// (4 x 8,192 of 12 heads of 64: 2,850 against 2,960).
template <typename T, int DP, bool kBias>
struct DqShape {
  static constexpr int kBlocks = sizeof(T) == 2 && DP <= 64 && !kBias ? 2 : 1;
  static constexpr int kTile = 32 * kBlocks;
  static constexpr int kBufs = 2;
  static constexpr int kBytes = 2 * kBufs * kTile * kPitch<DP> * (int)sizeof(T);
};
constexpr int kAttnWaves = kAttnThreads / 64;
// A row of the dS block: 32 values, then at least 31 zeros, and 4 words that spread the
// rows' 16-byte stores over the banks; 32 zeros stand before the first row.
constexpr int kDiagRow = 68, kDiagRows = 16;
constexpr int kDiagWords = kDiagRows * kDiagRow + 32;

// Adds the diagonals of half of the wave's block (rows: packed rows from `first_row`, the half
// starting at row `from`; columns: keys from `base`) to the wave's sums by relative position.
__device__ __forceinline__ void add_diagonals(const AttnArgs& a, const float* block, float* sums,
                                              int first_row, int from, int base, int pos0,
                                              int lane) {
  const int G = a.G;
  // relative position of (row 0, key 0) as an entry of the sums
  const int entry = base - pos0 + a.distance + kAttnPad;
  if (G == 1) {
    // diagonals key - (row - from) = -15 .. 31
    const float* p = block + lane - (kDiagRows - 1);
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kDiagRows; ++i) t += p[i * (kDiagRow + 1)];
    if (lane < 31 + kDiagRows) sums[entry - from + lane - (kDiagRows - 1)] += t;
    return;
  }
  // rows of head g: every G-th, their queries one apart
  const int rows = (30 + G) / G + 1;  // at most, counted from row 0's query
  const int wide = 31 + rows;         // diagonals of a head
  const int tok0 = query_of(a, first_row);
  for (int x = lane; x < G * wide; x += 64) {
    const int g = x / wide, diag = x - g * wide - (rows - 1);
    float t = 0.f;
    // first row of head g at or after the half's first
    const int start = first_row + from, tok = query_of(a, start);
    int r = g - (start - tok * G);
    if (r < 0) r += G;
    for (int i = query_of(a, start + r) - tok0; r < kDiagRows; r += G, ++i) {
      const int key = diag + i;
      if (key >= 0 && key < 32) t += block[r * kDiagRow + key];
    }
    sums[g * a.span + entry + diag] += t;
  }
}

// Order of a wave's own LDS writes and reads.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename T, int DP, bool kBias, bool kVec>
__global__ __launch_bounds__(kAttnThreads, (kGroupsPerCu<T, DP>)) void attn_dq_kernel(
    AttnArgs a) {
  using Shape = DqShape<T, DP, kBias>;
  constexpr int kBlocks = Shape::kBlocks, kTile = Shape::kTile;
  constexpr int kTileN = kTile * kPitch<DP>;
  constexpr bool kScaled = __is_same(T, f16);
  extern __shared__ __align__(16) uint8_t smem[];
  T* s_k = (T*)smem;
  T* s_v = s_k + Shape::kBufs * kTileN;
  float* s_bias = (float*)(smem + Shape::kBytes);
  float* s_diag = s_bias;                            // [wave][kDiagWords]
  float* s_far = s_diag;                             // [wave][half][32][2], after the keys
  if (kBias && a.dbias) s_bias = s_diag + kAttnWaves * kDiagWords;
  float* s_sum = s_bias + a.G * a.span;              // [wave][G][span]
  const AttnItem it = a.items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5;
  const int G = a.G, d = a.d;
  const LaneRow me = lane_row(a, it, it.row + wave * 32, lane);
  const float scale2 = a.scale * kLog2e;
  const bool wave_live = it.row + wave * 32 < it.nq * G;
  const bool want_bias = kBias && a.dbias;

  const T* k0 = (const T*)a.k.data + it.k0 * a.k.token_stride + it.kvh * a.k.head_stride;
  const T* v0 = (const T*)a.v.data + it.k0 * a.v.token_stride + it.kvh * a.v.head_stride;
  const uint8_t* mask = a.key_mask ? a.key_mask + it.k0 : nullptr;
  KeyStage<T, DP, kTile, kVec, kVec> stage;
  stage.place(a);
  uint8_t ok[kBlocks];
  auto fetch = [&](int base, int b) {
    stage.load(a, mask, k0, v0, base, it.hi, s_k + b * kTileN, s_v + b * kTileN);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
      if (mask || base + kTile > it.hi) ok[i] = key_ok(mask, base + 32 * i + (lane & 31), it.hi);
  };
  if (it.lo < it.hi) fetch(it.lo, 0);

  const int64_t at = (it.q0 + me.tok) * a.heads + it.kvh * G + me.g;
  // Where a row's keys fit one block, D is summed from P dP there: the output is rounded, which
  // costs short rows more than the rounding of dS.
  const bool one_block = it.hi <= 32 && it.hi > 0;
  // a row that saw no key has lse = -infinity; as +infinity it makes every P 0
  float lse2 = INFINITY, dsum = 0.f;
  vec8<T> q[DP / 16], dout[DP / 16];
  {
    const float lse = me.live ? a.lse[at] : -INFINITY;
    const T* pq = (const T*)a.q.data + (me.live ? row_at(a, a.q, it, me.r) : 0);
    const T* pd = (const T*)a.dout.data + (me.live ? row_at(a, a.dout, it, me.r) : 0);
    const T* po = (const T*)a.o.data + (me.live ? row_at(a, a.o, it, me.r) : 0);
    vec8<T> out[DP / 16];
    load_frags<T, DP, kVec>(pq, me.live, d, h, q);
    load_frags<T, DP, kVec>(pd, me.live, d, h, dout);
    load_frags<T, DP, kVec>(po, me.live, d, h, out);
    const bool some = lse != -INFINITY;
    if (some) lse2 = lse * kLog2e - kUpIn<T>;
    if (!__all(some)) {  // rows without keys, whatever they hold
#pragma unroll
      for (int c = 0; c < DP / 16; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          q[c][j] = some ? q[c][j] : (T)0.f;
          dout[c][j] = some ? dout[c][j] : (T)0.f;
        }
    }
#pragma unroll
    for (int c = 0; c < DP / 16; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) dsum += (float)dout[c][j] * (float)out[c][j];
    if (!some) dsum = 0.f;
    dsum += other_half(dsum);
    if (me.live && h == 0) a.dsum[at] = dsum;
  }
  float lo = 0.f, hi = 0.f, far_lo = 0.f, far_hi = 0.f;
  const float* table = nullptr;
  float *sums = nullptr, *block = nullptr;
  int range0 = 0, range1 = 0;
  if constexpr (kBias) {
    load_bias<T>(a, it.kvh, s_bias);
    if (want_bias) {
      for (int i = threadIdx.x; i < kAttnWaves * G * a.span; i += kAttnThreads) s_sum[i] = 0.f;
      for (int i = threadIdx.x; i < kAttnWaves * kDiagWords / 4; i += kAttnThreads)
        ((f32x4*)s_diag)[i] = f32x4{};
    }
    __syncthreads();
    table = s_bias + me.g * a.span;
    lo = table[0];
    hi = table[a.span - 1];
    sums = s_sum + wave * G * a.span;
    block = s_diag + wave * kDiagWords + 32;
    if (want_bias && (int)threadIdx.x >> 3 < G * a.nb) {
      const int b = ((int)threadIdx.x >> 3) % a.nb;
      range0 = a.range[2 * b];
      range1 = a.range[2 * b + 1];
    }
  }
  f32x16 dq[DP / 32];
#pragma unroll
  for (int b = 0; b < DP / 32; ++b) dq[b] = f32x16{};
  const lds_addr k_al = lds_of(s_k) + lane_along<T, DP>(lane);
  const lds_addr k_ac = lds_of(s_k) + lane_across<T, DP>(lane);
  bool odd = false;                  // the wave's dQ has to be done again (careful_row)
  float most = 0.f;                  // largest |dS| of the row so far, times 2^kUp
  float up = kScaled ? 0x1p16f : 1;  // and is rounded times this

  int buf = 0;
  if (it.lo < it.hi) {
    stage.store(mask, s_k, s_v);
    __syncthreads();
  }
  for (int base = it.lo; base < it.hi; base += kTile) {
    uint32_t bits[kBlocks], any = 0;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      bits[b] = mask || base + kTile > it.hi ? (uint32_t)__ballot(ok[b] != 0) : ~0u;
      if (a.causal) bits[b] &= upto(me.pos, base + 32 * b);
      any |= bits[b];
    }
    const bool more = base + kTile < it.hi;
    if (more) fetch(base + kTile, buf ^ 1);
    if (wave_live && __any(any != 0)) {
      const lds_addr sk = k_al + buf * kTileN * (int)sizeof(T);
      const lds_addr sv = sk + (lds_addr)((s_v - s_k) * sizeof(T));
      const lds_addr sk_ac = k_ac + buf * kTileN * (int)sizeof(T);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
          if (sizeof(T) == 4 && 16 * c >= d) break;
          s = mma(frag_along<T, DP>(sk, 32 * b, c), q[c], s);
          dp = mma(frag_along<T, DP>(sv, 32 * b, c), dout[c], dp);
        }
        const int first = base + 32 * b;
        finish_scores<kBias>(s, scale2, table, a.distance, me.pos, me.pos_min, me.pos_max, lo, hi,
                             first, h, bits[b], &dp);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[r] = exp2_up<T>(kBias ? s[r] - lse2 : s[r] * scale2 - lse2);
        if (b == 0 && one_block) {
          float t = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) t += s[r] == 0.f ? 0.f : s[r] * dp[r];
          dsum = (t + other_half(t)) * kUpOut;
          if (me.live && h == 0) a.dsum[at] = dsum;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= dp[r] - dsum;  // dS
        if constexpr (kBias) {
          if (want_bias) {
            if (first - me.pos_max >= a.distance || first + 31 - me.pos_min <= -a.distance) {
              float t = 0.f;
#pragma unroll
              for (int r = 0; r < 16; ++r) t += s[r];
              if (first > me.pos_min) far_hi += t;
              else far_lo += t;
            } else {
              // rows past the sequence's end have dS = 0
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                if ((lane >> 4 & 1) == half) {
#pragma unroll
                  for (int g = 0; g < 4; ++g)
                    *(f32x4*)(block + (lane & 15) * kDiagRow + 8 * g + 4 * h) =
                        f32x4{s[4 * g], s[4 * g + 1], s[4 * g + 2], s[4 * g + 3]};
                }
                wave_sync();
                add_diagonals(a, block, sums, it.row + wave * 32, half * 16, first, me.pos_min,
                              lane);
                wave_sync();
              }
            }
          }
        }
        if constexpr (kScaled) {
          float t = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) t = fmaxf(t, fabsf(s[r]));
          t = fmaxf(t, other_half(t));
          most = fmaxf(most, t);
          if (__any(most * up >= 0x1p15f)) {
            // the largest so far to 2^13 .. 2^14
            const float next =
                most * up >= 0x1p15f
                    ? __builtin_amdgcn_ldexpf(1.f, 14 - __builtin_amdgcn_frexp_expf(most))
                    : up;
            const float f = next / up;
            up = next;
#pragma unroll
            for (int e = 0; e < DP / 32; ++e)
#pragma unroll
              for (int r = 0; r < 16; ++r) dq[e][r] *= f;
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= up;
        }
        if (a.causal && !__all(bits[b] == ~0u)) odd |= odd_values<T, DP>(sk_ac, 32 * b);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const vec8<T> p = frag_of<T>(s, c);
#pragma unroll
          for (int e = 0; e < DP / 32; ++e)
            dq[e] = mma(frag_across<T, DP>(sk_ac, 32 * b + 16 * c, 32 * e), p, dq[e]);
        }
      }
    }
    if (more) {
      buf ^= 1;
      stage.store(mask, s_k + buf * kTileN, s_v + buf * kTileN);
      __syncthreads();
    }
  }
  if (__builtin_expect(odd, 0)) {
    const int first = it.row + wave * 32;
    for (int i = 0; i < 32 && first + i < it.nq * G; ++i) {
      float acc[2];
      float m_ = __shfl(lse2, i) + kUpIn<T>, l_ = __shfl(dsum, i);
      careful_row<T, kBias, true>(a, it, s_bias, first + i, lane, acc, m_, l_);
#pragma unroll
      for (int e = 0; e < (DP + 63) / 64; ++e)
        if (lane + 64 * e < d)
          ((T*)a.dq.data + row_at(a, a.dq, it, first + i))[lane + 64 * e] =
              (T)(acc[e] * a.scale);
    }
  } else if (me.live)
    store_row<T, DP, kVec>((T*)a.dq.data + row_at(a, a.dq, it, me.r), dq,
                           a.scale / up * kUpOut, d, h);
  if constexpr (kScaled) {
    if (!(most < INFINITY)) most = 0.f;  // such a row has no say in how the others are scaled
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    float* s_max = (float*)smem;
    __syncthreads();  // the last tile has been read
    if (lane == 0) s_max[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0)
      a.part_max[(int64_t)it.kvh * a.row_tiles + it.part] =
          fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])) * kUpOut;
  }
  if constexpr (kBias) {
    if (!want_bias) return;
    if (!me.live) far_lo = far_hi = 0.f;
    if (G == 1) {  // the wave's rows are one head's: lane 0 takes the sum
#pragma unroll
      for (int o = 32; o; o >>= 1) {
        far_lo += __shfl_xor(far_lo, o);
        far_hi += __shfl_xor(far_hi, o);
      }
    }
    __syncthreads();
    s_far[(wave * 64 + h * 32 + (lane & 31)) * 2] = far_lo;
    s_far[(wave * 64 + h * 32 + (lane & 31)) * 2 + 1] = far_hi;
    __syncthreads();
    const int all = G * a.span;
    for (int i = threadIdx.x; i < all; i += kAttnThreads) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) t += s_sum[w * all + i];
      s_sum[i] = t;  // entry i belongs to this thread alone
    }
    __syncthreads();
    // 8 threads a bucket
    float* to = a.part_bias + ((int64_t)it.kvh * a.row_tiles + it.part) * G * a.nb;
    const int sub = threadIdx.x & 7;
    for (int i = threadIdx.x >> 3; i < G * a.nb; i += kAttnThreads / 8) {
      const int g = i / a.nb, b = i - g * a.nb;
      int from = range0, to_entry = range1;  // of the first bucket, loaded at the start
      if (i >= kAttnThreads / 8) {
        from = a.range[2 * b];
        to_entry = a.range[2 * b + 1];
      }
      // the first and the last entry stand for what lies past the distance
      const bool has_lo = from == 0 && to_entry > 0, has_hi = to_entry == a.span;
      float t = 0.f;
      for (int e = from + sub; e < to_entry; e += 8) t += s_sum[g * a.span + e];
      if (has_lo || has_hi) {
        if (G == 1) {
          if (sub < kAttnWaves)
            t += (has_lo ? s_far[sub * 128] : 0.f) + (has_hi ? s_far[sub * 128 + 1] : 0.f);
        } else {
          // copy `sub` of the sums past the distance: the rows of this head
          const int row0 = it.row + (sub >> 1) * 32;
          int row = g - (row0 - query_of(a, row0) * G);
          if (row < 0) row += G;
          for (; row < 32; row += G) {
            if (has_lo) t += s_far[(sub * 32 + row) * 2];
            if (has_hi) t += s_far[(sub * 32 + row) * 2 + 1];
          }
        }
      }
#pragma unroll
      for (int o = 4; o; o >>= 1) t += __shfl_xor(t, o);
      if (sub == 0) to[i] = t * kUpOut;
    }
  }
}

// ---- backward: dK and dV -------------------------------------------------------------------
// A wave takes 32 of the tile's 128 keys, one a lane, and goes through the rows that see
// them: all query heads of the group, so that the sum over a shared head is the accumulator's.
// S = Q K^T puts rows 8 g + 4 h + t in registers 4 g + t.  The first `heads` work-groups of a
// launch with a bias's gradient add up its partial sums instead.  Issue bounds it: the two
// causal documents above 647 us (and 25 to join), the 256 documents 368.

template <typename T, int DP>
struct DkvShape {
  static constexpr int kBlocks = sizeof(T) == 2 && DP <= 64 ? 2 : 1;  // 32-row blocks of a tile
  static constexpr int kTile = 32 * kBlocks;
  static constexpr int kBufs = 2;
  static constexpr int kTileBytes = kTile * kPitch<DP> * (int)sizeof(T);
  // Chunks of 16 of the keys' and the values' operands that stay in registers.  The others are
  // in LDS: with them the accumulators would not fit two waves a SIMD (where the loop ran with
  // registers spilled to memory, each read of which waits for the next tile's loads: 2 x 8,192
  // tokens of 16 heads, backward, 4.5 ms with all chunks of K in registers, 3.7 with five).
  static constexpr int kChunks = DP / 16;
  static constexpr int kKeptV = DP * sizeof(T) >= 256 ? 0 : kChunks;
  static constexpr int kKeptK = DP == 128 && sizeof(T) == 2 ? 5 : kChunks;
  static constexpr int kWaveBytes = (2 * kChunks - kKeptK - kKeptV) * kFragBytes<T>;
  static constexpr int kValueBytes = kAttnThreads / 64 * kWaveBytes;
  static constexpr int kOddBytes = 16;  // of each buffer: whether its rows hold odd values
  static constexpr int kBytes =
      kValueBytes + kBufs * (2 * kTileBytes + 4 * kTile * 4) + kOddBytes;
};

template <typename T>
__device__ __forceinline__ void reduce_bias(const AttnArgs& a, int head, float* s) {
  // threads: nb / 2 pairs of buckets (rounded up to a power of two) x groups of row tiles
  int wide = 2;
  while (wide < a.nb / 2) wide *= 2;
  const int groups = kAttnThreads / wide, b = threadIdx.x % wide, g = threadIdx.x / wide;
  const int kvh = head / a.G;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const int64_t first = (int64_t)kvh * a.row_tiles * a.G + (head - kvh * a.G);
  const f32x2* p = (const f32x2*)(a.part_bias + first * a.nb) + b;
  const int64_t step = (int64_t)a.G * a.nb / 2;
  f32x2 t = {};
  if (2 * b < a.nb) {
#pragma unroll 8
    for (int i = g; i < a.row_tiles; i += groups) t += p[i * step];
  }
  ((f32x2*)s)[threadIdx.x] = t;
  __syncthreads();
  if (g == 0 && 2 * b < a.nb) {
    t = f32x2{};
    for (int i = 0; i < groups; ++i) t += ((f32x2*)s)[i * wide + b];
    ((T*)a.dbias)[(int64_t)(2 * b) * a.heads + head] = (T)t[0];
    ((T*)a.dbias)[(int64_t)(2 * b + 1) * a.heads + head] = (T)t[1];
  }
}

template <typename T, int DP, bool kBias, bool kVec>
__global__ __launch_bounds__(kAttnThreads, (kGroupsPerCu<T, DP>)) void attn_dkv_kernel(
    AttnArgs a) {
  using Shape = DkvShape<T, DP>;
  constexpr int kBlocks = Shape::kBlocks, kTile = Shape::kTile;
  constexpr int kTileN = kTile * kPitch<DP>;
  constexpr bool kScaled = __is_same(T, f16);
  extern __shared__ __align__(16) uint8_t smem[];
  // P is computed, and rounded, times 1 / kUpPOut
  constexpr bool kStartAtRow = sizeof(T) == 2;
  constexpr float kUpPIn = kScaled ? 14.f : kUpIn<T>, kUpPOut = kScaled ? 0x1p-14f : kUpOut;
  const int reducers = (int)gridDim.x - a.nitems;
  if (kBias && (int)blockIdx.x < reducers) {
    reduce_bias<T>(a, blockIdx.x, (float*)smem);
    return;
  }
  T* s_q = (T*)(smem + Shape::kValueBytes);
  T* s_do = s_q + Shape::kBufs * kTileN;
  // [buf][the row's exponent, -D, table offset, pos][row]
  float* s_row = (float*)(s_do + Shape::kBufs * kTileN);
  int* s_odd = (int*)(smem + Shape::kBytes - Shape::kOddBytes);  // [buf]
  float* s_bias = (float*)(smem + Shape::kBytes);
  const AttnItem it = a.items[blockIdx.x - reducers];
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5;
  const int G = a.G, d = a.d, shift = it.nk - it.nq;
  const float scale2 = a.scale * kLog2e;
  const int key0 = it.row + wave * 32, key = key0 + (lane & 31);
  const bool wave_live = key0 < it.nk;
  const bool there = key < it.nk;
  const bool live = there && (!a.key_mask || a.key_mask[it.k0 + key] != 0);

  // Rows that saw no key are zeros whatever they hold: their lse tells, loaded with them.
  using Tile = Stage<T, DP, kTile, kVec, kVec>;
  Tile st_q, st_do;
  constexpr int kN = Tile::kN;
  float piece_lse[kN], row_lse = 0.f, row_d = 0.f;
  int row_off = 0, row_pos = 0;
  bool row_there = false;
  const float* lse0 = a.lse + it.q0 * a.heads + it.kvh * G;  // the sequence's first row
  const float* dsum0 = a.dsum + it.q0 * a.heads + it.kvh * G;
  const T* q0 = (const T*)a.q.data + it.q0 * a.q.token_stride + it.kvh * G * a.q.head_stride;
  const T* do0 =
      (const T*)a.dout.data + it.q0 * a.dout.token_stride + it.kvh * G * a.dout.head_stride;
  // Offsets of a tile's pieces and rows from its first query.  Where G divides the tile they
  // are the same for every tile.
  const bool fixed = (G & (G - 1)) == 0 && G <= 32;
  const bool row_mine = threadIdx.x < kTile;
  // a row without keys is only possible with a mask or a table that holds -infinity
  const bool some_empty = a.key_mask || kBias;
  int off_lse[kN], off_row = 0, tok_row = 0;
  auto offsets = [&](int base) {
    const int tok0 = query_of(a, base);
    auto in = [&](const sieve_heads& x, int row, int col) {
      const int r = base + row, tok = query_of(a, r);
      return (tok - tok0) * x.token_stride + (r - tok * G) * x.head_stride + col;
    };
    st_q.place([&](int row, int col) { return in(a.q, row, col); }, d);
    st_do.place([&](int row, int col) { return in(a.dout, row, col); }, d);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int r = base + Tile::row(i), tok = query_of(a, r);
      off_lse[i] = (tok - tok0) * a.heads + (r - tok * G);
    }
    const int r = base + (int)threadIdx.x, tok = query_of(a, r);
    tok_row = tok - tok0;
    off_row = tok_row * a.heads + (r - tok * G);
    if (kBias) row_off = (r - tok * G) * a.span;
  };
  auto fetch = [&](int base, int b) {
    if (!fixed) offsets(base);
    const int tok0 = query_of(a, base);
    st_q.load(q0 + tok0 * a.q.token_stride, it.hi - base, d, s_q + b * kTileN);
    st_do.load(do0 + tok0 * a.dout.token_stride, it.hi - base, d, s_do + b * kTileN);
    const float* lse = lse0 + (int64_t)tok0 * a.heads;
    if (some_empty) {
#pragma unroll
      for (int i = 0; i < kN; ++i)
        piece_lse[i] = base + Tile::row(i) < it.hi ? lse[off_lse[i]] : -INFINITY;
    }
    if (row_mine) {
      row_lse = -INFINITY;
      row_d = 0.f;
      row_pos = tok0 + tok_row + shift;
      row_there = base + (int)threadIdx.x < it.hi;
      if (row_there) {
        row_lse = lse[off_row];
        row_d = (dsum0 + (int64_t)tok0 * a.heads)[off_row];
      }
    }
  };
  offsets(it.lo);
  auto put = [&](int b) {
    if (Tile::kDirectLoads) wait_loads();
    st_q.store(s_q + b * kTileN, some_empty, [&](int i) { return piece_lse[i] != -INFINITY; });
    st_do.store(s_do + b * kTileN, some_empty, [&](int i) { return piece_lse[i] != -INFINITY; });
    if (row_mine) {
      float* p = s_row + b * 4 * kTile + threadIdx.x;
      p[0] = row_lse == -INFINITY ? -INFINITY
                                  : (kUpPIn - row_lse * kLog2e) / (kStartAtRow ? scale2 : 1.f);
      p[kTile] = -row_d;
      ((int*)p)[2 * kTile] = row_off;
      ((int*)p)[3 * kTile] = row_pos;
    }
    // Infinities and NaN in a row's q or dout reach its lse or D.  A row of scores of -infinity
    // alone is cleared above where that may come of a mask or the bias.
    if (a.causal && wave == 0) {
      const bool bad = !(row_lse < INFINITY) || !(fabsf(row_d) < INFINITY) ||
                       (row_lse == -INFINITY && row_there && !some_empty);
      const bool any = __any(bad);
      if (lane == 0) s_odd[b] = any;
    }
  };
  if (it.lo < it.hi) fetch(it.lo, 0);

  const lds_addr q_al = lds_of(s_q) + lane_along<T, DP>(lane);
  const lds_addr q_ac = lds_of(s_q) + lane_across<T, DP>(lane);
  // chunks of the values, then of the keys
  const lds_addr kept = lds_of(smem) + wave * Shape::kWaveBytes + lane * 16;
  constexpr int kKeptK = Shape::kKeptK, kKeptV = Shape::kKeptV, kMoreV = Shape::kChunks - kKeptV;
  vec8<T> k[DP / 16], v[DP / 16];
  {
    const int64_t tok = it.k0 + (live ? key : 0);
    const T* pk = (const T*)a.k.data + tok * a.k.token_stride + it.kvh * a.k.head_stride;
    const T* pv = (const T*)a.v.data + tok * a.v.token_stride + it.kvh * a.v.head_stride;
    load_frags<T, DP, kVec>(pk, live, d, h, k);
    load_frags<T, DP, kVec>(pv, live, d, h, v);
#pragma unroll
    for (int c = kKeptV; c < DP / 16; ++c) keep_frag<T>(kept, c - kKeptV, v[c]);
#pragma unroll
    for (int c = kKeptK; c < DP / 16; ++c) keep_frag<T>(kept, kMoreV + c - kKeptK, k[c]);
  }
  if constexpr (kBias) load_bias<T>(a, it.kvh, s_bias);
  float up = 1.f;  // what brings dS times 1 / kUpPOut to where it is rounded
  if constexpr (kScaled) {
    float most = 0.f;
    const float* p = a.part_max + (int64_t)it.kvh * a.row_tiles + it.tile0;
    for (int i = lane; i < it.ntiles; i += 64) most = fmaxf(most, p[i]);
#pragma unroll
    for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    const int e = most > 0.f ? 14 - __builtin_amdgcn_frexp_expf(most) : 0;
    up = __builtin_amdgcn_ldexpf(kUpPOut, e < 40 ? e : 40);
  }
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int b = 0; b < DP / 32; ++b) dk[b] = dv[b] = f32x16{};
  bool odd = false;  // the wave's keys have to be done again (careful_key)

  int buf = 0;
  if (it.lo < it.hi) put(0);
  __syncthreads();
  for (int base = it.lo; base < it.hi; base += kTile) {
    const bool more = base + kTile < it.hi;
    if (more) fetch(base + kTile, buf ^ 1);
    if (wave_live) {
      constexpr int kApart = Shape::kBufs * kTileN * (int)sizeof(T);  // s_do - s_q
      lds_addr sq = q_al + buf * kTileN * (int)sizeof(T);
      lds_addr sq_ac = q_ac + buf * kTileN * (int)sizeof(T);
      // Work the reads' addresses out at each tile: kept over the loop they would fill the
      // registers that the accumulators leave.
      if constexpr (kMoreV > 0) asm volatile("" : "+v"(sq), "+v"(sq_ac));
      const lds_addr sd = sq + kApart, sd_ac = sq_ac + kApart;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const int first = base + 32 * b;
        const int last = (first + 31 < it.hi ? first + 31 : it.hi - 1);
        if (first >= it.hi) continue;
        const int pos_min = query_of(a, first) + shift, pos_max = query_of(a, last) + shift;
        if (a.causal && pos_max < key0) continue;
        const float* rows = s_row + buf * 4 * kTile + 32 * b + 4 * h;
        // S - lse and dP - D: the products are added to what is subtracted (but for S in fp32,
        // where adding its products to a larger number would cost bits).  A row without keys
        // has -infinity there, and P = 0.
        f32x16 s, dp;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 x = *(const f32x4*)(rows + 8 * g);
          const f32x4 y = *(const f32x4*)(rows + kTile + 8 * g);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            s[4 * g + t] = kStartAtRow ? x[t] : 0.f;
            dp[4 * g + t] = y[t];
          }
        }
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
          if (sizeof(T) == 4 && 16 * c >= d) break;
          const vec8<T> key_c =
              c < kKeptK ? k[c] : frag_kept<T>(kept, kMoreV + c - kKeptK);
          const vec8<T> val_c = c < kKeptV ? v[c] : frag_kept<T>(kept, c - kKeptV);
          s = mma(frag_along<T, DP>(sq, 32 * b, c), key_c, s);
          dp = mma(frag_along<T, DP>(sd, 32 * b, c), val_c, dp);
        }
        if constexpr (kBias) {
          const int dist = a.distance;
          if (G == 1 && (key0 - pos_max >= dist || key0 + 31 - pos_min <= -dist)) {
            const float far = s_bias[key0 > pos_min ? a.span - 1 : 0];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = s[r] * scale2 + far;
          } else if (G == 1) {
            // row 8 g + 4 h + t of the block stands at first + shift + that
            const float* table =
                s_bias + (key - (first + shift) - 4 * h + dist + kAttnPad) - 27;
#pragma unroll
            for (int r = 0; r < 16; ++r)
              s[r] = s[r] * scale2 + table[27 - 8 * (r >> 2) - (r & 3)];
          } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const i32x4 off = *(const i32x4*)(rows + 2 * kTile + 8 * g);
              const i32x4 pos = *(const i32x4*)(rows + 3 * kTile + 8 * g);
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                int rel = key - pos[t];
                rel = rel < -dist ? -dist : rel > dist ? dist : rel;
                s[4 * g + t] = s[4 * g + t] * scale2 + s_bias[off[t] + rel + dist + kAttnPad];
              }
            }
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= scale2;
        }
        if constexpr (!kStartAtRow) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 x = *(const f32x4*)(rows + 8 * g);
#pragma unroll
            for (int t = 0; t < 4; ++t) s[4 * g + t] += x[t];
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = exp2_up<T>(s[r]);
        if (a.causal && pos_min < key0 + 31) {
          odd |= __builtin_amdgcn_readfirstlane(s_odd[buf]) != 0;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const i32x4 pos = *(const i32x4*)(rows + 3 * kTile + 8 * g);
#pragma unroll
            for (int t = 0; t < 4; ++t)
              if (key > pos[t]) s[4 * g + t] = dp[4 * g + t] = 0.f;
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dp[r] *= s[r];
          if constexpr (kScaled) dp[r] *= up;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const vec8<T> p = frag_of<T>(s, c), ds = frag_of<T>(dp, c);
#pragma unroll
          for (int e = 0; e < DP / 32; ++e) {
            dv[e] = mma(frag_across<T, DP>(sd_ac, 32 * b + 16 * c, 32 * e), p, dv[e]);
            dk[e] = mma(frag_across<T, DP>(sq_ac, 32 * b + 16 * c, 32 * e), ds, dk[e]);
          }
        }
      }
    }
    if (more) {
      buf ^= 1;
      put(buf);
      __syncthreads();
    }
  }
  if (__builtin_expect(odd, 0)) {
    const AttnArgs c = args_again();
    const AttnItem item = c.items[blockIdx.x - ((int)gridDim.x - c.nitems)];
    for (int i = 0; i < 32 && key0 + i < item.nk; ++i) {
      float ck[2] = {}, cv[2] = {};
      const int64_t tok = item.k0 + key0 + i;
      if (!c.key_mask || c.key_mask[tok] != 0)
        careful_key<T, kBias>(c, item, s_bias, key0 + i, lane, ck, cv);
      T* to_k = (T*)c.dk.data + tok * c.dk.token_stride + item.kvh * c.dk.head_stride;
      T* to_v = (T*)c.dv.data + tok * c.dv.token_stride + item.kvh * c.dv.head_stride;
      const int64_t slot = (int64_t)item.part * 2 * kAttnKeys + wave * 32 + i;
#pragma unroll
      for (int e = 0; e < (DP + 63) / 64; ++e) {
        const int col = lane + 64 * e;
        if (item.part >= 0) {
          if (col < DP) {
            c.part_kv[slot * DP + col] = ck[e] * c.scale;
            c.part_kv[(slot + kAttnKeys) * DP + col] = cv[e];
          }
        } else if (col < c.d) {
          to_k[col] = (T)(ck[e] * c.scale);
          to_v[col] = (T)cv[e];
        }
      }
    }
    return;
  }
  if (!there) return;
  if (!live) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dk[b] = dv[b] = f32x16{};
  }
  if (it.part >= 0) {
    float* p = a.part_kv + ((int64_t)it.part * 2 * kAttnKeys + wave * 32 + (lane & 31)) * DP;
    const float fk = a.scale / up * kUpPOut, fv = kUpPOut;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * b + 8 * g + 4 * h;
        *(f32x4*)(p + col) = f32x4{dk[b][4 * g] * fk, dk[b][4 * g + 1] * fk,
                                   dk[b][4 * g + 2] * fk, dk[b][4 * g + 3] * fk};
        *(f32x4*)(p + kAttnKeys * DP + col) =
            f32x4{dv[b][4 * g] * fv, dv[b][4 * g + 1] * fv, dv[b][4 * g + 2] * fv,
                  dv[b][4 * g + 3] * fv};
      }
    return;
  }
  const int64_t tok = it.k0 + key;
  store_row<T, DP, kVec>((T*)a.dk.data + tok * a.dk.token_stride + it.kvh * a.dk.head_stride, dk,
                   a.scale / up * kUpPOut, d, h);
  store_row<T, DP, kVec>((T*)a.dv.data + tok * a.dv.token_stride + it.kvh * a.dv.head_stride, dv,
                   kUpPOut, d, h);
}

// Partial sums of one key tile to its gradients, kDkvJoinGroups work-groups a tile.
constexpr int kDkvJoinGroups = 8;

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads) void attn_dkv_join_kernel(AttnArgs a) {
  const AttnJoin j = a.joins[blockIdx.x / kDkvJoinGroups];
  constexpr int kAll = 2 * kAttnKeys * DP / 4;  // values, four a thread
  constexpr int kEach = kAll / kDkvJoinGroups;
  const int first = blockIdx.x % kDkvJoinGroups * kEach;
  for (int i = first + threadIdx.x; i < first + kEach; i += kAttnThreads) {
    const int col = i % (DP / 4) * 4, key = j.row + i / (DP / 4) % kAttnKeys;
    if (key >= j.n || col >= a.d) continue;
    f32x4 v = {};
    const f32x4* p = (const f32x4*)a.part_kv + (int64_t)j.part0 * kAll + i;
#pragma unroll 4
    for (int n = 0; n < j.parts; ++n) v += p[(int64_t)n * kAll];
    const sieve_heads& to = i < kAll / 2 ? a.dk : a.dv;
    T* t = (T*)to.data + (j.t0 + key) * to.token_stride + j.kvh * to.head_stride + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < a.d) t[e] = (T)v[e];
  }
}

// ---- launch ----------------------------------------------------------------------------------

constexpr int kMaxLds = 160 * 1024;

template <void (*kKernel)(AttnArgs)>
hipError_t launch(const AttnArgs& a, int grid, size_t lds, hipStream_t s) {
  if (lds > kMaxLds) return hipErrorInvalidValue;
  if (lds > 64 * 1024) {  // more has to be asked for, once for each kernel and device
    static std::atomic<uint64_t> done{0};
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    e = once_per_device(done, device, [] {
      return hipFuncSetAttribute((const void*)kKernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                 kMaxLds);
    });
    if (e != hipSuccess) return e;
  }
  kKernel<<<grid, kAttnThreads, lds, s>>>(a);
  return hipGetLastError();
}

template <typename T, int DP, bool kBias, bool kVec>
hipError_t launch_as(AttnKind kind, const AttnArgs& a, int grid, hipStream_t s) {
  const size_t table = kBias ? (size_t)a.G * a.span * sizeof(float) : 0;
  switch (kind) {
    case kAttnFwd:
      return launch<attn_forward_kernel<T, DP, 1, kBias, kVec>>(
          a, grid, FwdShape<T, DP, 1>::kBytes + table, s);
    case kAttnFwdFew:
      return launch<attn_forward_kernel<T, DP, 4, kBias, kVec>>(
          a, grid, FwdShape<T, DP, 4>::kBytes + table, s);
    case kAttnDq: {
      const size_t sums = a.dbias ? kAttnWaves * (table + kDiagWords * sizeof(float)) : 0;
      return launch<attn_dq_kernel<T, DP, kBias, kVec>>(
          a, grid, DqShape<T, DP, kBias>::kBytes + table + sums, s);
    }
    case kAttnDkv:
      return launch<attn_dkv_kernel<T, DP, kBias, kVec>>(
          a, grid, DkvShape<T, DP>::kBytes + table, s);
    default:
      return hipErrorInvalidValue;
  }
}

template <typename T, int DP>
hipError_t launch_dp(AttnKind kind, const AttnArgs& a, int grid, hipStream_t s) {
  constexpr int kJoin = (kAttnRows + kJoinRows<DP> - 1) / kJoinRows<DP>;
  constexpr int kJoinFew = (kAttnFewRows + kJoinRows<DP> - 1) / kJoinRows<DP>;
  if (kind == kAttnDkvJoin)
    return launch<attn_dkv_join_kernel<T, DP>>(a, grid * kDkvJoinGroups, 0, s);
  if (kind == kAttnJoin)
    return launch<attn_join_kernel<T, DP, kAttnRows>>(a, grid * kJoin, 0, s);
  if (kind == kAttnJoinFew)
    return launch<attn_join_kernel<T, DP, kAttnFewRows>>(a, grid * kJoinFew, 0, s);
  if (a.bias)
    return a.vec ? launch_as<T, DP, true, true>(kind, a, grid, s)
                 : launch_as<T, DP, true, false>(kind, a, grid, s);
  return a.vec ? launch_as<T, DP, false, true>(kind, a, grid, s)
               : launch_as<T, DP, false, false>(kind, a, grid, s);
}

template <typename T>
hipError_t launch_type(AttnKind kind, int dp, const AttnArgs& a, int grid, hipStream_t s) {
  if (grid <= 0) return hipSuccess;
  switch (dp) {
    case 32: return launch_dp<T, 32>(kind, a, grid, s);
    case 64: return launch_dp<T, 64>(kind, a, grid, s);
    case 96: return launch_dp<T, 96>(kind, a, grid, s);
    case 128: return launch_dp<T, 128>(kind, a, grid, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace
}  // namespace sieve
