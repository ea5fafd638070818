// orth.hip -- a stack of matrices made nearly orthogonal by a polynomial iteration, as an
// optimizer does with the momentum of a layer's weights.
//
//   X = G / (|G| + eps),  then `steps` times  X <- B X,  B = a I + b A + c A A,  A = X X^T
//
// (with |G| the root of the sum of squares; matrices taller than wide: A = X^T X, X <- X B).  Each
// step maps every singular value s of X to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// A step is three products and nothing else: A = X X^T with C = b I + c A in its epilogue, then
// B = a I + A C, then B X, whose accumulators are the next X.  A, C and B are symmetric: only the
// tiles on and below the diagonal are computed, those below it written to both sides.
//
// What is weak in G is multiplied by up to a^steps (484 for the usual five), and rounding errors
// with it, so 16-bit values are not enough between the products, whatever G's type is.  Every
// matrix is kept as two binary16 parts, hi = round(v), lo = round(v - hi): 24 bits together, and
// a product is hi hi + hi lo + lo hi, summed in fp32.  That is fp32's precision at a third of
// the 16-bit rate, 5 times the fp32 matrix rate.  Nothing multiplies what the last step leaves, so
// a bfloat16 result's has the hi parts alone (kPlainSteps).  All values are bounded by singular
// values, so fixed powers of two keep them in binary16's range (kScaleX, kScaleA): |X| below 4,
// |A|, |B| and |C| below 16, which the host checks for the coefficients that it is given.
//
// Its products bound it from some 768 x 768 on, launches below.  Measured, five steps: one of
// 256 x 256 114 us, 17 kernels of 3 to 9 us; 36 of 768 x 768 bf16 1.60 ms; 8 of 1,024 x 4,096 f32
// 2.31 ms, of which a step's X takes 227 us (910 TFLOP/s of 16-bit products), A 191, B 55.  C is
// written beside A, as tiles of B that computed it from A's in their epilogue took longer.
#include <math.h>

#include <algorithm>

#include "mm_tile.h"
#include "once_per_device.h"

using namespace sieve;

namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kThreads = 256;
// A work-group's tile: the usual one at two work-groups a CU; one for few tiles, which are bound
// by the latency of their loads, with more of these on their way.
template <int kSide_, int kStep, int kStages, int kPlanes_>
struct Shape {
  static constexpr int kSide = kSide_, kPlanes = kPlanes_;
  template <bool kAcrossA, bool kAcrossB>
  using Tile = MmTile<mm_f16, kSide, kSide, kAcrossA, kAcrossB, 2, 2, kStep, kStages, kPlanes>;
  static constexpr int kLds = Tile<false, false>::kLds;
};
// of both parts, and of the first alone
typedef Shape<128, 32, 2, 2> Usual;
typedef Shape<64, 32, 4, 2> Few;
typedef Shape<128, 64, 2, 1> UsualPlain;
typedef Shape<64, 64, 4, 1> FewPlain;
constexpr float kScaleX = 16384.f, kScaleA = 4096.f;  // of X; of A and B
constexpr double kMaxX = 3.9, kMaxA = 15.9;           // below 65504 times these
constexpr int kMaxSide = 65536;
constexpr int kMaxSteps = 1000;
// Of the last steps, for bfloat16: 36 of 768 x 768 in 1,632 us, the error 1.12 times that of
// rounding the exact result; with none 1,838 us and 1.00 times, with two 1.4 times at 98% of the
// time.
constexpr int kPlainSteps = 1;
constexpr int kSums = 64;                             // parts of a matrix's sum of squares
// Up to so many tiles of the usual shape leave half of the CUs idle, and are computed in four times
// as many small ones.  fp32, five steps, with small tiles and without: 256 x 256 114 us and 220,
// 1,024 x 1,024 262 and 512, two of them 357 and 521; with all small ones and by this rule: 4 of
// 1,024 x 1,024 602 us and 537, 2,048 x 2,048 1,092 and 932.
constexpr int64_t kFewTiles = 128;
constexpr int64_t kMostBytes = int64_t(1) << 31;      // of the workspace, for one matrix or more

struct Source {
  const void* g;
  int64_t batch_stride, row_stride;
  int64_t m, n, pitch;
  float eps;
  double* sums;          // [matrix][kSums]
  f16* x;                // [plane][matrix][m][pitch]
  int64_t plane;
  void* out;             // without steps: the result
};

// 8 values of a row from a column that is a multiple of 8, zeros past its end.
template <typename T, bool kWhole>
__device__ __forceinline__ void load8(const T* row, int col, int n, float (&v)[8]) {
  if constexpr (kWhole) {
    const EncVec<T, 8> q = enc_load<T, 8>(row + col);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)q.v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = col + j < n ? (float)row[col + j] : 0.f;
  }
}

// A work-group's parts of a matrix: moves blockIdx.x * 256 + thread, and so on, by gridDim.x * 256.
// f(row, column of 8)
template <typename F>
__device__ __forceinline__ void each_move(const Source& a, F f) {
  const uint32_t moves = (uint32_t)(a.pitch / 8);
  const uint64_t all = (uint64_t)a.m * moves;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all;
       i += (uint64_t)gridDim.x * 256) {
    // fewer than 2^16 x 2^13 moves
    const uint32_t row = (uint32_t)i / moves;
    f((int)row, (int)((uint32_t)i - row * moves) * 8);
  }
}

template <typename T, bool kWhole>
__global__ __launch_bounds__(256) void orth_norm_kernel(Source a) {
  __shared__ double s[4];
  const T* g = (const T*)a.g + blockIdx.y * a.batch_stride;
  double sum = 0.0;
  each_move(a, [&](int row, int col) {
    float v[8];
    load8<T, kWhole>(g + row * a.row_stride, col, (int)a.n, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fma((double)v[j], (double)v[j], sum);
  });
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) a.sums[blockIdx.y * kSums + blockIdx.x] = s[0] + s[1] + s[2] + s[3];
}

__device__ __forceinline__ void split(float v, f16& hi, f16& lo) {
  hi = (f16)v;
  lo = (f16)(v - (float)hi);
}

// X of the matrix, zeros up to the pitch.
template <typename T, bool kWhole, bool kOut>
__global__ __launch_bounds__(256) void orth_scale_kernel(Source a) {
  __shared__ double s_inv;
  if (threadIdx.x < 64) {
    double sum = a.sums[blockIdx.y * kSums + threadIdx.x];
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (threadIdx.x == 0) s_inv = 1.0 / (sqrt(sum) + (double)a.eps);
  }
  __syncthreads();
  const double inv = s_inv;
  const T* g = (const T*)a.g + blockIdx.y * a.batch_stride;
  each_move(a, [&](int row, int col) {
    float v[8];
    load8<T, kWhole>(g + row * a.row_stride, col, (int)a.n, v);
    const int64_t matrix_row = blockIdx.y * a.m + row;
    if constexpr (kOut) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j < a.n) ((T*)a.out)[matrix_row * a.n + col + j] = (T)(float)(v[j] * inv);
    } else {
      EncVec<f16, 8> hi, lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) split((float)(v[j] * inv) * kScaleX, hi.v[j], lo.v[j]);
      enc_store<f16, 8>(a.x + matrix_row * a.pitch + col, hi);
      enc_store<f16, 8>(a.x + a.plane + matrix_row * a.pitch + col, lo);
    }
  });
}
static_assert(kSums == 64, "a wave adds up the parts");

// One product of a step, for every matrix.
struct Product {
  MmOperand a, b;        // of the first matrix
  int64_t a_next, b_next;
  int64_t k;
  int64_t rows, cols;    // that are written: zeros past the matrix's, up to the pitch
  int64_t side;
  uint32_t tiles, tiles_m, tiles_n;  // tiles of a matrix
  uint32_t all;
  float fa, fb, fc;      // the coefficients
  void* out;             // planes or the result
  void* second;          // b I + c A, with A
  int64_t pitch, next, plane;
};

enum { kGram, kPolynomial, kUpdate, kLast };

// The tiles of every matrix's product.
template <int kKind, int kSide>
struct Tiles {
  MmPlaces at;
  uint32_t tiles, tiles_m, tiles_n;
  int64_t k;
  __device__ __forceinline__ explicit Tiles(const Product& a)
      : at(a.all), tiles(a.tiles), tiles_m(a.tiles_m), tiles_n(a.tiles_n), k(a.k) {}
  __device__ __forceinline__ void get(MmWork& w, int64_t& matrix) const {
    matrix = at.place / tiles;
    const uint32_t in = at.place % tiles;
    uint32_t tm, tn;
    if constexpr (kKind == kGram || kKind == kPolynomial) {
      // tiles on and below the diagonal, row by row
      tm = (uint32_t)((sqrtf(8.f * in + 1.f) - 1.f) * 0.5f);
      while (tm * (tm + 1) / 2 > in) --tm;
      while ((tm + 1) * (tm + 2) / 2 <= in) ++tm;
      tn = in - tm * (tm + 1) / 2;
    } else {
      mm_tile_at(in, tiles_m, tiles_n, 8, tm, tn);
    }
    w = {(int64_t)tm * kSide, (int64_t)tn * kSide, 0, k};
  }
};

template <typename T, int kKind, typename S, bool kAcrossA, bool kAcrossB>
__global__ __launch_bounds__(kThreads, 2) void orth_product_kernel(Product a) {
  extern __shared__ __attribute__((aligned(1024))) char lds_memory[];
  typedef typename S::template Tile<kAcrossA, kAcrossB> Tile;
  Tiles<kKind, S::kSide> tiles(a);
  // one tile a work-group: matrices lie apart
  MmWork w;
  int64_t matrix;
  tiles.get(w, matrix);
  MmOperand x = a.a, y = a.b;
  x.p = (const f16*)x.p + matrix * a.a_next;
  y.p = (const f16*)y.p + matrix * a.b_next;
  Tile t(x, y, 1,
         (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)lds_memory);
  bool first_one = true;
  auto next = [&](MmWork& to) {
    to = w;
    const bool was = first_one;
    first_one = false;
    return was;
  };
  t.start(next);
  t.sum(t.steps_of(w), next);
  const int64_t at = matrix * a.next + w.m0 * a.pitch + w.n0;
  const int64_t rows = a.rows - w.m0, cols = a.cols - w.n0;
  if constexpr (kKind == kLast) {
    const MmPatch<T> to((T*)a.out + at, a.pitch, rows, cols);
#pragma unroll
    for (int j = 0; j < Tile::kJ; ++j) {
      const auto lane = to.lane(t.row0, t.col0 + 32 * j);
#pragma unroll
      for (int i = 0; i < Tile::kI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          to.store(to.at(lane, Tile::down(i, r)),
                   (T)(t.acc[i][j][r] * (1.f / (kScaleA * kScaleX))));
    }
    t.stop();
    return;
  }
  const bool plain = S::kPlanes == 1;  // what is multiplied next has first parts alone, too
  const MmPatch<f16> hi((f16*)a.out + at, a.pitch, rows, cols);
  const MmPatch<f16> lo((f16*)a.out + a.plane + at, a.pitch, rows, cols);
  // A and B below the diagonal also go to the other side of it; tiles on it are whole
  const int64_t other = matrix * a.next + w.n0 * a.pitch + w.m0;
  const bool mirrored = kKind != kUpdate && w.m0 != w.n0;
  const MmPatch<f16> hi2((f16*)a.out + other, a.pitch, mirrored ? cols : 0, rows);
  const MmPatch<f16> lo2((f16*)a.out + a.plane + other, a.pitch, mirrored ? cols : 0, rows);
  // and with A goes b I + c A
  f16* second = (f16*)a.second;
  const MmPatch<f16> hi3(second + at, a.pitch, rows, cols);
  const MmPatch<f16> lo3(second + a.plane + at, a.pitch, rows, cols);
  const MmPatch<f16> hi4(second + other, a.pitch, mirrored ? cols : 0, rows);
  const MmPatch<f16> lo4(second + a.plane + other, a.pitch, mirrored ? cols : 0, rows);
#pragma unroll
  for (int j = 0; j < Tile::kJ; ++j) {
    const int col = t.col0 + 32 * j;
    const int odd = (int)threadIdx.x & 1;
    const auto lane = hi.lane(t.row0 + odd, col - odd);
    const int64_t gap = w.n0 + col - w.m0 - t.row0;  // rows down to the diagonal
    const int diagonal = w.n0 + col < a.side && gap >= 0 && gap < S::kSide ? (int)gap : -1;
#pragma unroll
    for (int i = 0; i < Tile::kI; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f16 h[4], l[4], h3[4], l3[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = Tile::down(i, 4 * g + e);
          float v = t.acc[i][j][4 * g + e];
          if constexpr (kKind == kGram) v *= kScaleA / (kScaleX * kScaleX);
          else v *= 1.f / kScaleA;
          if constexpr (kKind == kPolynomial) v += d == diagonal ? a.fa * kScaleA : 0.f;
          split(v, h[e], l[e]);
          if constexpr (kKind == kGram)
            split(a.fc * v + (d == diagonal ? a.fb * kScaleA : 0.f), h3[e], l3[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const uint32_t o = hi.at(lane, Tile::down(i, 4 * g + e));
          hi.store_rows(o, h[e], h[e + 1]);
          if (!plain) lo.store_rows(o, l[e], l[e + 1]);
          if constexpr (kKind == kGram) {
            hi3.store_rows(o, h3[e], h3[e + 1]);
            if (!plain) lo3.store_rows(o, l3[e], l3[e + 1]);
          }
        }
        if (mirrored) {
          // the lane's column is a row there, its 4 rows neighbours in it (all there, or none)
          const int d = Tile::down(i, 4 * g);
          const uint32_t o = t.row0 + d < hi2.cols && col < hi2.rows
                                 ? ((uint32_t)col * hi2.pitch + t.row0 + d) * 2 : kMmNowhere;
          hi2.store4(o, h);
          if (!plain) lo2.store4(o, l);
          if constexpr (kKind == kGram) {
            hi4.store4(o, h3);
            if (!plain) lo4.store4(o, l3);
          }
        }
      }
  }
  t.stop();
}

// ---- host ------------------------------------------------------------------------------------

int64_t round256(int64_t n) { return (n + 255) & ~int64_t(255); }

struct Layout {
  int64_t side, pitch, side_pitch;  // of A and B; of X's rows; of A's and B's rows
  int64_t batch;                    // matrices at a time
  int64_t sums, x[2], gram, second, poly, bytes;
};

Layout layout_of(int64_t batch, int64_t m, int64_t n) {
  Layout l{};
  l.side = std::min(m, n);
  l.pitch = (n + 7) & ~int64_t(7);
  l.side_pitch = (l.side + 7) & ~int64_t(7);
  const int64_t one = 4 * (2 * m * l.pitch + 3 * l.side_pitch * l.side_pitch);
  // a launch's work-groups have fewer than 2^32 threads
  const int64_t tiles = ((m + 63) / 64) * ((n + 63) / 64);
  l.batch = std::max<int64_t>(1, std::min({batch, kMostBytes / one, (int64_t(1) << 23) / tiles,
                                           int64_t(65535)}));
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t was = at;
    at += round256(bytes);
    return was;
  };
  l.sums = take(l.batch * kSums * 8);
  for (int i = 0; i < 2; ++i) l.x[i] = take(l.batch * m * l.pitch * 4);
  l.gram = take(l.batch * l.side_pitch * l.side_pitch * 4);
  l.second = take(l.batch * l.side_pitch * l.side_pitch * 4);
  l.poly = take(l.batch * l.side_pitch * l.side_pitch * 4);
  l.bytes = at;
  return l;
}

// Whether all values stay in range: singular values start in [0, 1], and a step maps
// [0, s] into [0, max |p|] with p(x) = a x + b x^3 + c x^5; B's are p(x) / x.
bool in_range(double a, double b, double c, int steps) {
  double s = 1.0;
  for (int i = 0; i < steps; ++i) {
    auto p = [&](double x) { return fabs(x * (a + x * x * (b + x * x * c))); };
    auto q = [&](double x2) { return fabs(a + x2 * (b + x2 * c)); };
    double top = p(s), most = std::max(q(0.0), q(s * s));
    if (c != 0.0) {
      const double at = -b / (2.0 * c);
      if (at > 0.0 && at < s * s) most = std::max(most, q(at));
    }
    // p' = a + 3 b x^2 + 5 c x^4
    double roots[2] = {-1.0, -1.0};
    if (c != 0.0) {
      const double d = 9.0 * b * b - 20.0 * a * c;
      if (d >= 0.0) {
        roots[0] = (-3.0 * b + sqrt(d)) / (10.0 * c);
        roots[1] = (-3.0 * b - sqrt(d)) / (10.0 * c);
      }
    } else if (b != 0.0) {
      roots[0] = -a / (3.0 * b);
    }
    for (double r : roots)
      if (r > 0.0 && r < s * s) top = std::max(top, p(sqrt(r)));
    most = std::max({most, fabs(b), fabs(b + c * s * s)});  // of b I + c A
    if (!(s * s <= kMaxA && most <= kMaxA && top <= kMaxX)) return false;
    s = top;
  }
  return true;
}

int check_orth(int64_t batch, int64_t m, int64_t n) {
  if (batch < 0) return set_error(SIEVE_EINVAL, "batch is negative");
  if (m < 1 || n < 1) return set_error(SIEVE_EINVAL, "m and n must be >= 1");
  if (m > kMaxSide || n > kMaxSide)
    return set_error(SIEVE_EUNSUPPORTED, "m or n is above %d", kMaxSide);
  return SIEVE_OK;
}

static_assert(std::max({Usual::kLds, Few::kLds, UsualPlain::kLds, FewPlain::kLds}) <= 65536,
              "no larger LDS has to be asked for");

template <typename T>
void run(const void* g, int64_t batch_stride, int64_t row_stride, int64_t batch, int64_t m,
         int64_t n, int steps, const float* coefficients, float eps, void* out, char* w,
         const Layout& l, hipStream_t s) {
  const bool tall = m > n;
  Source src{g, batch_stride, row_stride, m, n, l.pitch, eps, (double*)(w + l.sums),
             (f16*)(w + l.x[0]), batch * m * l.pitch, out};
  const dim3 parts(kSums, (uint32_t)batch);
  // some 4 moves a thread
  const int64_t groups = (m * (l.pitch / 8) + 1023) / 1024;
  const dim3 rows((uint32_t)std::min<int64_t>(groups, 4096), (uint32_t)batch);
  const bool whole = n % 8 == 0 && ((uintptr_t)g & 15) == 0 && row_stride * sizeof(T) % 16 == 0 &&
                     batch_stride * sizeof(T) % 16 == 0;
  auto begin = [&](auto w8) {
    constexpr bool kWhole = decltype(w8)::value;
    orth_norm_kernel<T, kWhole><<<parts, 256, 0, s>>>(src);
    if (steps == 0) orth_scale_kernel<T, kWhole, true><<<rows, 256, 0, s>>>(src);
    else orth_scale_kernel<T, kWhole, false><<<rows, 256, 0, s>>>(src);
  };
  if (whole) begin(std::true_type{});
  else begin(std::false_type{});
  if (steps == 0) return;
  const int64_t side = l.side, sp = l.side_pitch, square = sp * sp;
  f16 *gram = (f16*)(w + l.gram), *second = (f16*)(w + l.second), *poly = (f16*)(w + l.poly);
  const MmOperand of_a{gram, sp, side, batch * square}, of_c{second, sp, side, batch * square},
      of_b{poly, sp, side, batch * square};
  bool plain = false;  // the first parts alone
  // the product's kernel with tiles of the shape that it asks for
  auto launch = [&](Product p, auto kind, auto across_a, auto across_b) {
    constexpr int kKind = decltype(kind)::value;
    constexpr bool kA = decltype(across_a)::value, kB = decltype(across_b)::value;
    constexpr bool kHalf = kKind == kGram || kKind == kPolynomial;
    auto with = [&](auto shape) {
      typedef decltype(shape) S;
      p.tiles_m = (uint32_t)((p.rows + S::kSide - 1) / S::kSide);
      p.tiles_n = (uint32_t)((p.cols + S::kSide - 1) / S::kSide);
      p.tiles = kHalf ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
      p.all = p.tiles * (uint32_t)batch;
      orth_product_kernel<T, kKind, S, kA, kB><<<p.all, kThreads, S::kLds, s>>>(p);
    };
    const int64_t tm = (p.rows + 127) / 128, tn = (p.cols + 127) / 128;
    const bool few = (kHalf ? tm * (tm + 1) / 2 : tm * tn) * batch <= kFewTiles;
    if constexpr (std::is_same_v<T, bf16> && kKind != kUpdate) {  // kUpdate: never the last
      if (plain) {
        if (few) with(FewPlain{});
        else with(UsualPlain{});
        return;
      }
    }
    if (few) with(Few{});
    else with(Usual{});
  };
  const std::integral_constant<bool, true> across;
  const std::integral_constant<bool, false> along;
  for (int i = 0; i < steps; ++i) {
    const f16* x = (const f16*)(w + l.x[i & 1]);
    f16* to = (f16*)(w + l.x[(i + 1) & 1]);
    const bool last = i == steps - 1;
    // A: over the longer side
    Product p{};
    plain = steps - i <= kPlainSteps;
    p.a = p.b = {x, l.pitch, side, src.plane};
    p.a_next = p.b_next = m * l.pitch;
    p.k = tall ? m : n;
    p.rows = p.cols = sp;
    p.side = side;
    p.fa = coefficients[0];
    p.fb = coefficients[1];
    p.fc = coefficients[2];
    p.out = gram;
    p.second = second;
    p.pitch = sp;
    p.next = square;
    p.plane = batch * square;
    const std::integral_constant<int, kGram> gram_kind;
    if (tall) launch(p, gram_kind, across, across);
    else launch(p, gram_kind, along, along);
    // B
    p.a = of_a;
    p.b = of_c;
    p.a_next = p.b_next = square;
    p.k = side;
    p.out = poly;
    launch(p, std::integral_constant<int, kPolynomial>{}, along, along);
    // the next X, or the result
    p.a = tall ? MmOperand{x, l.pitch, m, src.plane} : of_b;
    p.b = tall ? of_b : MmOperand{x, l.pitch, n, src.plane};
    p.a_next = tall ? m * l.pitch : square;
    p.b_next = tall ? square : m * l.pitch;
    p.rows = m;
    p.cols = last ? n : l.pitch;
    p.out = last ? out : (void*)to;
    p.pitch = last ? n : l.pitch;
    p.next = m * p.pitch;
    p.plane = src.plane;
    const std::integral_constant<int, kUpdate> update;
    const std::integral_constant<int, kLast> the_last;
    if (tall && last) launch(p, the_last, along, along);
    else if (tall) launch(p, update, along, along);
    else if (last) launch(p, the_last, along, across);
    else launch(p, update, along, across);
  }
}

}  // namespace

SIEVE_API int64_t sieve_orthogonalize_workspace(int64_t batch, int64_t m, int64_t n) {
  clear_error();
  if (int st = check_orth(batch, m, n)) return st;
  return batch ? layout_of(batch, m, n).bytes : 0;
}

SIEVE_API int sieve_orthogonalize(const void* g, int64_t batch_stride, int64_t row_stride,
                                  int32_t dtype, int64_t batch, int64_t m, int64_t n,
                                  int32_t steps, const float* coefficients, float eps, void* x,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  if (!enc_dtype_ok(dtype))
    return set_error(SIEVE_EINVAL, "dtype = %d is not one of SIEVE_F32, SIEVE_F16, SIEVE_BF16",
                     dtype);
  if (int st = check_orth(batch, m, n)) return st;
  if (steps < 0) return set_error(SIEVE_EINVAL, "steps is negative");
  if (steps > kMaxSteps)
    return set_error(SIEVE_EUNSUPPORTED, "steps = %d is above %d", steps, kMaxSteps);
  if (!(eps >= 0.f) || eps == INFINITY)
    return set_error(SIEVE_EINVAL, "eps must be >= 0 and finite");
  if (!coefficients) return set_error(SIEVE_EINVAL, "coefficients must be non-NULL");
  for (int i = 0; i < 3; ++i)
    if (!isfinite(coefficients[i]))
      return set_error(SIEVE_EINVAL, "coefficients must be finite");
  if (!in_range(coefficients[0], coefficients[1], coefficients[2], steps))
    return set_error(SIEVE_EUNSUPPORTED,
                     "with these coefficients singular values in [0, 1] may grow past %g", kMaxX);
  if (batch == 0) return SIEVE_OK;
  if (!g || !x) return set_error(SIEVE_EINVAL, "g and x must be non-NULL");
  if (row_stride < n || batch_stride < 0)
    return set_error(SIEVE_EINVAL, "row_stride is below n, or batch_stride negative");
  const Layout l = layout_of(batch, m, n);
  if (!workspace || workspace_bytes < l.bytes || ((uintptr_t)workspace & 15))
    return set_error(SIEVE_EINVAL, "workspace must be 16-byte aligned and hold %lld bytes",
                     (long long)l.bytes);
  const int size = enc_size(dtype);
  for (int64_t z = 0; z < batch; z += l.batch) {
    const int64_t some = std::min(l.batch, batch - z);
    const char* from = (const char*)g + z * batch_stride * size;
    char* to = (char*)x + z * m * n * size;
    auto go = [&](auto t) {
      run<decltype(t)>(from, batch_stride, row_stride, some, m, n, steps, coefficients, eps, to,
                       (char*)workspace, l, (hipStream_t)stream);
    };
    if (dtype == SIEVE_F32) go(float{});
    else if (dtype == SIEVE_F16) go(f16{});
    else go(bf16{});
  }
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}
