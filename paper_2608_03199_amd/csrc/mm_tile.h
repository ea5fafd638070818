// mm_tile.h -- tiles of matrix products on the 16-bit matrix units, for the operators whose
// products end in something else than a store (loss.hip, orth.hip).
//
//   acc(m, n) = sum over k of A(m, k) B(n, k), in fp32
//
// Each operand lies in memory along k (its rows are m or n) or across it (its rows are k): no
// operand is transposed in memory.  Values of 32 bits come as planes of 16-bit parts, and the
// sum then runs over those pairs of planes whose product is above fp32's last bit.
//
// A work-group of four waves (2 x 2) owns BM x BN values, a wave a quarter of it in 32 x 32
// tiles.  Steps of 32 along k go through three LDS buffers: while one is read, the loads of the
// next two are on their way, straight into LDS.  Two work-groups share a CU, so that one's
// epilogue and waits lie under the other's products.
//
// LDS holds 16-byte pieces of an operand in the order of its memory rows, permuted within a
// row by the row's number so that the reads below touch every bank equally:
//   along k: 64 bytes a row; a read takes one piece of each of 32 rows;
//   across k: 2 BM bytes a row; a transposing read takes 4 rows by 16 columns a quarter wave.
#pragma once

#include <type_traits>

#include "enc_common.h"

namespace sieve {

typedef __bf16 mm_bf16;
typedef _Float16 mm_f16;
typedef float mm_f32x16 __attribute__((ext_vector_type(16)));
typedef short mm_s16x4 __attribute__((ext_vector_type(4)));
typedef int mm_i32x4 __attribute__((ext_vector_type(4)));

constexpr int64_t kMmMaxStride = 1 << 20;  // values: offsets within a tile stay below 2^31 bytes
constexpr uint32_t kMmNowhere = 0x80000000u;

// One operand: value (row, k) is p[row * stride + k], or p[k * stride + row] across k.  p and
// stride are multiples of 16 bytes, and so is what the contiguous axis may be read by: along k
// the values up to the next multiple of 8 are there and zero (or k ends at one), across k
// those of the rows are there, whatever they hold.
struct MmOperand {
  const void* p;
  int64_t stride;
  int64_t rows;    // of m or n
  int64_t plane;   // values between planes
};

// Pairs of planes, smallest products first: all six for three planes, the last three for two,
// the last for one.
__device__ __forceinline__ int mm_plane_a(int i) { return (0x001102 >> (4 * i)) & 15; }
__device__ __forceinline__ int mm_plane_b(int i) { return (0x010120 >> (4 * i)) & 15; }

template <typename T>
__device__ __forceinline__ mm_f32x16 mm_mfma(enc_u32x4 a, enc_u32x4 b, mm_f32x16 c) {
  typedef T v8 __attribute__((ext_vector_type(8)));
  if constexpr (std::is_same_v<T, mm_f16>)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a),
                                                  __builtin_bit_cast(v8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a),
                                                   __builtin_bit_cast(v8, b), c, 0, 0, 0);
}

template <int N>
__device__ __forceinline__ void mm_wait_loads() {
  static_assert(N < 64);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The wave's LDS reads have arrived, then the work-group's.  (__syncthreads would also wait for
// the loads that are to stay in flight.)
__device__ __forceinline__ void mm_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand's way into LDS, R rows of m or n, kStep values of k at a time.
template <int R, bool kAcross, int kStep, int kThreads>
struct MmStage {
  static constexpr int kBytes = R * kStep * 2;
  static constexpr int kLoads = kBytes / 16 / kThreads;  // of a thread
  static_assert(kBytes % (16 * kThreads) == 0 && (kStep == 32 || kStep == 64));
  static constexpr int kPitch = kAcross ? R * 2 : kStep * 2;  // bytes of a row
  static constexpr int kPieces = kPitch / 16;

  uint32_t off[kLoads];
  int k_first;  // of this thread's first piece; the others lie kKStep on
  static constexpr int kKStep = kAcross ? kThreads / kPieces : 0;

  // Which piece of row `row` lies at place c is c ^ turn(row).
  static __device__ __forceinline__ int turn(int row) {
    if constexpr (!kAcross) return kStep == 32 ? row >> 2 & 3 : row >> 1 & 7;
    else if constexpr (kPieces >= 16) return (row & 3) << 2 | (row >> 2 & 3);
    else return (row & 2) << 1 | (row >> 2 & 3);
  }

  __device__ __forceinline__ void place(const MmOperand& x, int64_t row0) {
    const int64_t left = x.rows - row0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * kThreads + (int)threadIdx.x;
      const int row = at / kPieces, piece = at % kPieces ^ turn(row);
      const uint32_t o = (uint32_t)(row * (uint32_t)x.stride + piece * 8) * 2;
      off[i] = (kAcross ? piece * 8 : row) < left ? o : kMmNowhere;
      if (i == 0) k_first = kAcross ? row : piece * 8;
    }
  }

  // Starts the loads of a step of which `left` values of k are there; base: the tile's first
  // value of the step; to: the LDS address of the buffer.
  __device__ __forceinline__ void load(const char* base, int left, uint32_t to) const {
    const uint64_t b = (uint64_t)base;
    const mm_i32x4 rsrc = {(int)(uint32_t)b, (int)(uint32_t)(b >> 32 & 0xffff), (int)kMmNowhere,
                           0x00027000};
    const uint32_t wave_to =
        to + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t o = k_first + i * kKStep < left ? off[i] : kMmNowhere;
      // no register is written: what arrives is waited for by count, before the barrier in
      // front of the step that reads it
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   ::"s"(wave_to + i * kThreads * 16), "v"(o), "s"(rsrc)
                   : "memory");
    }
  }

  // A lane's place in a buffer for frag(): row0 is the wave's first row, a multiple of 32.
  static __device__ __forceinline__ uint32_t lane_at(int row0) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    if constexpr (kAcross) {
      // rows (k) 8 half + (i / 4), columns 16 (q & 1) + 4 (i & 3) of quarter q's lane i
      const int i = lane & 15, k = 8 * half + (i >> 2);
      const int piece = row0 / 8 + (lane >> 3 & 2) + (i >> 1 & 1);
      return k * kPitch + ((piece ^ turn(k)) * 16) + (i & 1) * 8;
    } else {
      const int row = row0 + (lane & 31);
      return row * kPitch + ((half ^ turn(row)) * 16);
    }
  }
  // Values k = 16 s + 8 (lane / 32) .. + 7 of row 32 j + lane % 32 from the wave's first.
  // at: the buffer's address plus lane_at.
  static __device__ __forceinline__ enc_u32x4 frag(uint32_t at, int j, int s) {
    if constexpr (kAcross) {
      typedef __attribute__((address_space(3))) mm_s16x4 lds_s16x4;
      union {
        mm_s16x4 half[2];
        enc_u32x4 all;
      } u;
      const uint32_t x = (at ^ (j * 64)) + s * 16 * kPitch;
      u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)x);
      // 4 rows on, turn differs in bit 0
      u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(uintptr_t)((x ^ 16) + 4 * kPitch));
      return u.all;
    } else {
      return *(const __attribute__((address_space(3))) enc_u32x4*)(uintptr_t)((at ^ (s * 32)) +
                                                                              j * 32 * kPitch);
    }
  }
};

// WM x WN waves own BM x BN values.
template <typename T, int BM, int BN, bool kAcrossA, bool kAcrossB, int WM = 2, int WN = 2,
          int kStep = 32, int kStages = 3>
struct MmTile {
  static constexpr int kThreads = 64 * WM * WN;
  typedef MmStage<BM, kAcrossA, kStep, kThreads> A;
  typedef MmStage<BN, kAcrossB, kStep, kThreads> B;
  static constexpr int kI = BM / WM / 32, kJ = BN / WN / 32;
  static constexpr int kStage = A::kBytes + B::kBytes;
  static constexpr int kLds = kStages * kStage;
  static constexpr int kLoads = A::kLoads + B::kLoads;
  mm_f32x16 acc[kI][kJ];

  // Register r of tile (i, j) of a wave holds row row(i, r) and column col(j) of the
  // work-group's values.
  static __device__ __forceinline__ int row(int i, int r) {
    return (int)(threadIdx.x >> 6) / WN * (BM / WM) + i * 32 + (r >> 2) * 8 +
           (int)(threadIdx.x >> 5 & 1) * 4 + (r & 3);
  }
  static __device__ __forceinline__ int col(int j) {
    return (int)(threadIdx.x >> 6) % WN * (BN / WN) + j * 32 + (int)(threadIdx.x & 31);
  }

  // lds: the address of kLds bytes, a multiple of 1024; free again on return.
  __device__ __forceinline__ void run(const MmOperand& a, int64_t m0, const MmOperand& b,
                                      int64_t n0, int64_t k0, int64_t k1, int pairs,
                                      uint32_t lds) {
    A sa;
    B sb;
    sa.place(a, m0);
    sb.place(b, n0);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint32_t a_at = lds + A::lane_at(wave / WN * (BM / WM));
    const uint32_t b_at = lds + A::kBytes + B::lane_at(wave % WN * (BN / WN));
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const int steps = (int)((k1 - k0 + kStep - 1) / kStep) * pairs;
    if (steps <= 0) return;
    int64_t k = k0;
    int pair = 6 - pairs;
    // past the last step nothing is there: the loads are counted all the same
    auto load = [&](int buffer) {
      const int left = pair < 6 ? (int)(k1 - k < kStep ? k1 - k : kStep) : 0;
      const int p = pair < 6 ? pair : 5;
      const int64_t at_a =
          mm_plane_a(p) * a.plane + (kAcrossA ? k * a.stride + m0 : m0 * a.stride + k);
      const int64_t at_b =
          mm_plane_b(p) * b.plane + (kAcrossB ? k * b.stride + n0 : n0 * b.stride + k);
      sa.load((const char*)a.p + at_a * 2, left, lds + buffer * kStage);
      sb.load((const char*)b.p + at_b * 2, left, lds + buffer * kStage + A::kBytes);
      k += kStep;
      if (k >= k1) {
        k = k0;
        ++pair;
      }
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) load(i);
    int buffer = 0;
    for (int step = 0; step < steps; ++step) {
      mm_wait_loads<(kStages - 2) * kLoads>();  // this step's; the next ones' stay in flight
      mm_barrier();
      load(buffer == 0 ? kStages - 1 : buffer - 1);
      const uint32_t at = buffer * kStage;
#pragma unroll
      for (int s = 0; s < kStep / 16; ++s) {
        enc_u32x4 fa[kI], fb[kJ];
#pragma unroll
        for (int j = 0; j < kJ; ++j) fb[j] = B::frag(b_at + at, j, s);
#pragma unroll
        for (int i = 0; i < kI; ++i) fa[i] = A::frag(a_at + at, i, s);
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int j = 0; j < kJ; ++j) acc[i][j] = mm_mfma<T>(fa[i], fb[j], acc[i][j]);
      }
      buffer = buffer == kStages - 1 ? 0 : buffer + 1;
    }
    mm_wait_loads<0>();
    mm_barrier();
  }
};

// The place of a work-group among `all`: consecutive work-groups go to the chip's eight dies in
// turn, each with an L2 of its own, so a die takes a run of places.
__device__ __forceinline__ uint32_t mm_place_of(uint32_t index, uint32_t all) {
  const uint32_t each = all / 8, more = all % 8, die = index % 8;
  return die * each + (die < more ? die : more) + index / 8;
}

// The tile at a place: runs go through `high` tiles of m before the next of n.
__device__ __forceinline__ void mm_tile_at(uint32_t place, uint32_t tiles_m, uint32_t tiles_n,
                                           uint32_t high, uint32_t& tm, uint32_t& tn) {
  const uint32_t strip = high * tiles_n;
  const uint32_t s = place / strip, in = place % strip;
  const uint32_t rows = tiles_m - s * high < high ? tiles_m - s * high : high;
  tm = s * high + in % rows;
  tn = in / rows;
}

}  // namespace sieve
