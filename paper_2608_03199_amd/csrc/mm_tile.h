// mm_tile.h -- tiles of matrix products on the 16-bit matrix units, for the operators whose
// products end in something else than a store (loss.hip, orth.hip).
//
//   acc(m, n) = sum over k of A(m, k) B(n, k), in fp32
//
// Each operand lies in memory along k (its rows are m or n) or across it (its rows are k): no
// operand is transposed in memory.  Values of more than 16 bits come as planes of 16-bit parts,
// and the sum then takes those pairs of planes whose product is above fp32's last bit: three of
// two planes, six of three.  A step's planes are in LDS together, so that each is read once for
// all of its products.
//
// A work-group's waves share BM x BN values, in 32 x 32 tiles.  Steps along k go through LDS
// buffers: while one is read, the loads of the next are on their way, straight into LDS.
//
// LDS holds 16-byte pieces of an operand in the order of its memory rows, permuted within a
// row by the row's number so that the reads below touch every bank equally:
//   along k: a step's values a row; a read takes one piece of each of 32 rows;
//   across k: 2 BM bytes a row; a transposing read takes 4 rows by 16 columns a quarter wave.
//
// 8,192^3 bf16, both along k, 256 x 256 tiles, steps of 64, two buffers: 891 us, 1,234 TFLOP/s
// (with 256 x 128, steps of 32 and three buffers 1,189 us).
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

#pragma clang diagnostic push
// m0 is named as written all the same: nothing may be kept in it across the loads
#pragma clang diagnostic ignored "-Winline-asm"
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
    const mm_i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)b),
                           __builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32 & 0xffff)),
                           (int)kMmNowhere, 0x00027000};
    const uint32_t wave_to = (uint32_t)__builtin_amdgcn_readfirstlane(
        (int)(to + (threadIdx.x >> 6) * 1024));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t o = k_first + i * kKStep < left ? off[i] : kMmNowhere;
      // no register is written: what arrives is waited for by count, before the barrier in
      // front of the step that reads it
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   ::"s"(wave_to + i * kThreads * 16), "v"(o), "s"(rsrc)
                   : "m0", "memory");
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

#pragma clang diagnostic pop

// One tile's share of a product.
struct MmWork {
  int64_t m0, n0;   // its first row of A and of B
  int64_t k0, k1;   // the values of k that it sums
};

// The places of a work-group among `all` tiles that the whole grid shares out.  Consecutive
// work-groups go to the chip's eight dies in turn, each with an L2 of its own, so a die takes a
// run of places, and its work-groups take them side by side.
struct MmPlaces {
  uint32_t place, end, step;
  // before: tiles that were shared out the same way just before these: the work-groups that had
  // one more of them come last now
  __device__ __forceinline__ explicit MmPlaces(uint32_t all, uint32_t before = 0) {
    const uint32_t die = blockIdx.x % 8, each = all / 8, more = all % 8;
    const uint32_t first = die * each + (die < more ? die : more);
    const uint32_t had = before / 8 + (die < before % 8 ? 1 : 0);
    end = first + each + (die < more ? 1 : 0);
    step = (gridDim.x - die + 7) / 8;
    const uint32_t slot = blockIdx.x / 8, skip = had % step;
    place = first + (slot >= skip ? slot - skip : slot + step - skip);
  }
  __device__ __forceinline__ bool there() const { return place < end; }
  __device__ __forceinline__ void next() { place += step; }
};
// Work-groups for `all` tiles where `most` fit on the chip at once.
inline uint32_t mm_grid(uint64_t all, uint32_t most) {
  return (uint32_t)(all < most ? all : most);
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

// A pointer that is the same in all lanes, known to be.
template <typename V>
__device__ __forceinline__ V* mm_uniform(V* p) {
  const uint64_t b = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32));
  return (V*)((uint64_t)hi << 32 | lo);
}

// A tile's values in memory: rows x cols of them are there; loads of the others give zeros, and
// stores are dropped, without a branch.  pitch: values between rows, 256 of which span less than
// 2^31 bytes.
template <typename V>
struct MmPatch {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t pitch;
  int rows, cols;
  __device__ __forceinline__ MmPatch(V* first, int64_t pitch_, int64_t rows_, int64_t cols_)
      : rsrc(__builtin_amdgcn_make_buffer_rsrc(mm_uniform(first), 0, (int)kMmNowhere, 0x00027000)),
        pitch((uint32_t)pitch_), rows((int)(rows_ < 65536 ? rows_ : 65536)),
        cols((int)(cols_ < 65536 ? cols_ : 65536)) {}
  // A lane's place: a row and a column, and what is left of the rows from there.
  struct Lane {
    uint32_t base;
    int left;
  };
  __device__ __forceinline__ Lane lane(int row, int col) const {
    const uint32_t o = ((uint32_t)row * pitch + (uint32_t)col) * (uint32_t)sizeof(V);
    return {col < cols ? o : kMmNowhere, rows - row};
  }
  // d rows on.  What is added to kMmNowhere leads nowhere, too.
  __device__ __forceinline__ uint32_t at(const Lane& l, int d) const {
    const uint32_t o = l.base + (uint32_t)d * pitch * (uint32_t)sizeof(V);
    return d < l.left ? o : kMmNowhere;
  }
  __device__ __forceinline__ V load(uint32_t at) const {
    static_assert(sizeof(V) == 4);
    return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)at, 0, 0));
  }
  __device__ __forceinline__ void store(uint32_t at, V v) const {
    if constexpr (sizeof(V) == 4)
      __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), rsrc, (int)at, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), rsrc, (int)at, 0, 0);
  }
  // A row's value v0 and the next row's v1 of every lane's column, two neighbours of a row a store:
  // even lanes store the row's, odd ones the next row's.  at: of lane(row + odd, column - odd).
  __device__ __forceinline__ void store_rows(uint32_t at, V v0, V v1) const {
    static_assert(sizeof(V) == 2);
    const bool odd = threadIdx.x & 1;
    const uint32_t a = __builtin_bit_cast(uint16_t, v0), b = __builtin_bit_cast(uint16_t, v1);
    // what the neighbour stores goes there, what this lane stores comes (quad_perm 1 0 3 2)
    const uint32_t came = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(odd ? a : b), 0xb1, 0xf,
                                                                0xf, true);
    const uint32_t d = odd ? came | b << 16 : a | came << 16;
    __builtin_amdgcn_raw_buffer_store_b32(d, rsrc, (int)at, 0, 0);
  }
  // 4 neighbours of a row, at a multiple of 8 bytes
  __device__ __forceinline__ void store4(uint32_t at, const V (&v)[4]) const {
    static_assert(sizeof(V) == 2);
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    u32x2 d;
    __builtin_memcpy(&d, v, 8);
    __builtin_amdgcn_raw_buffer_store_b64(d, rsrc, (int)at, 0, 0);
  }
};

// WM x WN waves own BM x BN values at a time.  A work-group goes through its tiles as through one
// long sum: the first steps of the next tile are on their way while a tile's epilogue runs.
// kPlanes: of both operands, or 1, and then `planes_b` of B's in turn.
template <typename T, int BM, int BN, bool kAcrossA, bool kAcrossB, int WM, int WN, int kStep,
          int kStages, int kPlanes = 1>
struct MmTile {
  static constexpr int kThreads = 64 * WM * WN;
  typedef MmStage<BM, kAcrossA, kStep, kThreads> A;
  typedef MmStage<BN, kAcrossB, kStep, kThreads> B;
  static constexpr int kI = BM / WM / 32, kJ = BN / WN / 32;
  static constexpr int kStage = kPlanes * (A::kBytes + B::kBytes);
  static constexpr int kLds = kStages * kStage;
  static constexpr int kLoads = kPlanes * (A::kLoads + B::kLoads);
  mm_f32x16 acc[kI][kJ];

  // Register r of tile (i, j) of a wave holds row row0 + down(i, r) and column col0 + 32 j of the
  // work-group's values.
  int row0, col0;
  static __device__ __forceinline__ constexpr int down(int i, int r) {
    return i * 32 + (r >> 2) * 8 + (r & 3);
  }
  static __device__ __forceinline__ int wave() {
    return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  }

  const MmOperand &a, &b;
  const int planes_b;
  const uint32_t lds;
  A sa;
  B sb;
  MmWork ahead;     // the tile whose steps are being loaded, and where in it
  int64_t k;
  int plane;        // of B, the last one first; -1: nothing is left
  int buffer = 0;   // of the next step to be multiplied
  uint32_t a_at, b_at;

  // lds: the address of kLds bytes, a multiple of 1024, that nothing else uses.
  __device__ __forceinline__ MmTile(const MmOperand& a_, const MmOperand& b_, int planes_b_,
                                    uint32_t lds_)
      : a(a_), b(b_), planes_b(kPlanes == 1 ? planes_b_ : 1), lds(lds_) {
    const int wave_row = wave() / WN * (BM / WM), wave_col = wave() % WN * (BN / WN);
    a_at = lds + A::lane_at(wave_row);
    b_at = lds + kPlanes * A::kBytes + B::lane_at(wave_col);
    row0 = wave_row + (int)(threadIdx.x >> 5 & 1) * 4;
    col0 = wave_col + (int)(threadIdx.x & 31);
  }

  // Starts the next step's loads.  next(w): the work of the tile after the one that was loaded
  // last, false where there is none.
  template <typename Next>
  __device__ __forceinline__ void load(int to, Next& next) {
    // past the last step nothing is there: the loads are counted all the same
    const bool there = plane >= 0;
    const int left = there ? (int)(ahead.k1 - k < kStep ? ahead.k1 - k : kStep) : 0;
    const int64_t at_a = kAcrossA ? k * a.stride + ahead.m0 : ahead.m0 * a.stride + k;
    const int64_t at_b = (kAcrossB ? k * b.stride + ahead.n0 : ahead.n0 * b.stride + k) +
                         (there ? plane : 0) * b.plane;
    const uint32_t at = lds + to * kStage;
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
      sa.load((const char*)a.p + (at_a + p * a.plane) * 2, left, at + p * A::kBytes);
      sb.load((const char*)b.p + (at_b + p * b.plane) * 2, left,
              at + kPlanes * A::kBytes + p * B::kBytes);
    }
    if (!there) return;
    k += kStep;
    if (k >= ahead.k1) {
      k = ahead.k0;
      if (--plane < 0) begin(next);
    }
  }
  template <typename Next>
  __device__ __forceinline__ void begin(Next& next) {
    MmWork w;
    while (next(w)) {
      if (w.k0 >= w.k1) continue;  // no steps: see steps_of
      ahead = w;
      k = w.k0;
      plane = planes_b - 1;
      sa.place(a, w.m0);
      sb.place(b, w.n0);
      return;
    }
  }
  __device__ __forceinline__ int steps_of(const MmWork& w) const {
    return w.k1 > w.k0 ? (int)((w.k1 - w.k0 + kStep - 1) / kStep) * planes_b : 0;
  }

  // Starts the loads of the first tile's first steps; the work-group has one at least.
  template <typename Next>
  __device__ __forceinline__ void start(Next& next) {
    ahead = {0, 0, 0, 0};
    k = 0;
    plane = -1;
    sa.place(a, 0);
    sb.place(b, 0);
    begin(next);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) load(i, next);
  }

  // Sums a tile of so many steps into acc.
  template <typename Next>
  __device__ __forceinline__ void sum(int steps, Next& next) {
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    for (int step = 0; step < steps; ++step) {
      mm_wait_loads<(kStages - 2) * kLoads>();  // this step's; the next ones' stay in flight
      mm_barrier();
      load(buffer == 0 ? kStages - 1 : buffer - 1, next);
      const uint32_t at = buffer * kStage;
#pragma unroll
      for (int s = 0; s < kStep / 16; ++s) {
        enc_u32x4 fa[kPlanes][kI], fb[kPlanes][kJ];
#pragma unroll
        for (int p = 0; p < kPlanes; ++p) {
#pragma unroll
          for (int j = 0; j < kJ; ++j) fb[p][j] = B::frag(b_at + at + p * B::kBytes, j, s);
#pragma unroll
          for (int i = 0; i < kI; ++i) fa[p][i] = A::frag(a_at + at + p * A::kBytes, i, s);
        }
        // the smallest products first
#pragma unroll
        for (int both = kPlanes - 1; both >= 0; --both)
#pragma unroll
          for (int p = 0; p <= both; ++p)
#pragma unroll
            for (int i = 0; i < kI; ++i)
#pragma unroll
              for (int j = 0; j < kJ; ++j)
                acc[i][j] = mm_mfma<T>(fa[p][i], fb[both - p][j], acc[i][j]);
      }
      buffer = buffer == kStages - 1 ? 0 : buffer + 1;
    }
  }

  // What was loaded past the last tile has arrived: LDS may be given back.
  __device__ __forceinline__ void stop() { mm_wait_loads<0>(); }
};

}  // namespace sieve
