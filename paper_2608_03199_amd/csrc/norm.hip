// norm.hip -- layer norm over rows, forward and backward, with the residual sum
// in front of it and the reduction of the weights' gradients.
//
//   h = x + residual, u = (h - mean) rstd, y = u w + b
//   g = dy w, dx = rstd (g - mean(g) - u mean(g u)) + dh
//   dw = sum_rows dy u, db = sum_rows dy
//
// Each value is read once and written once, so memory bounds every kernel here but the looping
// ones.  65,536 x 1,024 bf16: forward 47 us, 5.7 TB/s; backward with its reduction 80 us, 5.0 TB/s,
// with dh 108.
// A row stays in the registers of a quarter of a wave (up to 128 values), a wave (up to
// 2,048) or a work-group (up to 8,192): the mean is taken first and the variance from the
// differences, in fp32 without the cancellation of a sum of squares.  Longer rows are read
// again, from the L2, by the looping kernels.
//
// The weights' gradients: a thread owns the same columns of every row it takes, so it
// sums them in registers; the work-group's rows add up through LDS,
// each work-group writes one partial row, and a second kernel adds those in a fixed
// order.  No atomics: equal calls give equal bits.
#include <type_traits>

#include "enc_common.h"

using namespace sieve;

namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxN = 65536;
constexpr int kMaxHeld = 8192;  // longest row that stays in registers
constexpr int kBigThreads = 1024;
// Work-groups of the backward pass: 2 a CU.  65,536 x 1,024 bf16 81 us, with 256 93, with 1,024
// 90; 65,536 x 768 f16 61, 78 and 59.
constexpr int kMaxParts = 512;

struct NormFwd {
  const void *x, *residual, *w, *b;
  int64_t x_stride, r_stride, rows;
  int n;
  float eps;
  void *y, *h;
  float *mean, *rstd;
};

struct NormBwd {
  const void *dy, *h, *w, *dh;
  const float *mean, *rstd;
  int64_t dy_stride, h_stride, rows;
  int n;
  void *dx, *dw, *db;
  float* part;  // [work-group][2][n]; null where there is one work-group
};

// Column of value e of a thread: E neighbours at a time (one move), or, where the rows are
// not aligned (E = 0), one neighbour a thread.
template <int NT, int E>
__device__ __forceinline__ int column(int e, int t) {
  return E ? ((e / (E ? E : 1)) * NT + t) * E + e % (E ? E : 1) : e * NT + t;
}

// E neighbours in moves of at most 16 bytes.
template <typename T, int E>
__device__ __forceinline__ EncVec<T, E> load_some(const T* p) {
  if constexpr (E * sizeof(T) >= 16) {
    return enc_load<T, E>(p);
  } else {
    return __builtin_bit_cast(EncVec<T, E>, *(const uint2*)p);
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_some(T* p, const EncVec<T, E>& v) {
  if constexpr (E * sizeof(T) >= 16)
    enc_store<T, E>(p, v);
  else
    *(uint2*)p = __builtin_bit_cast(uint2, v);
}

// Values of a row; 0 past its end.
template <typename T, int NE, int NT, int E>
__device__ __forceinline__ void load_row(const T* p, int n, int t, float (&v)[NE]) {
  if constexpr (E != 0) {
#pragma unroll
    for (int e = 0; e < NE; e += E) {
      const int col = column<NT, E>(e, t);
      if (col < n) {
        const EncVec<T, E> q = load_some<T, E>(p + col);
#pragma unroll
        for (int j = 0; j < E; ++j) v[e + j] = (float)q.v[j];
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) v[e + j] = 0.f;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const int col = column<NT, E>(e, t);
      v[e] = col < n ? (float)p[col] : 0.f;
    }
  }
}

// A row's values as they lie in memory, so that the next row can be on its way while one is
// worked on at half of the registers (or all, in 32 bits).
template <typename T, int NE, int NT, int E>
struct RawRow {
  T v[NE];

  __device__ __forceinline__ void load(const T* p, int n, int t) {
    if constexpr (E != 0) {
#pragma unroll
      for (int e = 0; e < NE; e += E) {
        const int col = column<NT, E>(e, t);
        if (col < n) {
          const EncVec<T, E> q = load_some<T, E>(p + col);
#pragma unroll
          for (int j = 0; j < E; ++j) v[e + j] = q.v[j];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const int col = column<NT, E>(e, t);
        if (col < n) v[e] = p[col];
      }
    }
  }
  __device__ __forceinline__ void get(int n, int t, float (&f)[NE]) const {
#pragma unroll
    for (int e = 0; e < NE; ++e) f[e] = column<NT, E>(e, t) < n ? (float)v[e] : 0.f;
  }
};

template <typename T, int NE, int NT, int E>
__device__ __forceinline__ void store_row(T* p, int n, int t, const float (&v)[NE]) {
  if constexpr (E != 0) {
#pragma unroll
    for (int e = 0; e < NE; e += E) {
      const int col = column<NT, E>(e, t);
      if (col < n) {
        EncVec<T, E> q;
#pragma unroll
        for (int j = 0; j < E; ++j) q.v[j] = (T)v[e + j];
        store_some<T, E>(p + col, q);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const int col = column<NT, E>(e, t);
      if (col < n) p[col] = (T)v[e];
    }
  }
}

// The sum over a row's threads within the wave.
template <int NT>
__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
  for (int o = (NT < 64 ? NT : 64) / 2; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Sums over the threads of a row: part of a wave, a wave, or the work-group through LDS.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* s) {
  v = lane_sum<NT>(v);
  if constexpr (NT > 64) {
    __syncthreads();  // the previous sum has been read
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) v += s[i];
  }
  return v;
}

template <int NT>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* s) {
  a = lane_sum<NT>(a);
  b = lane_sum<NT>(b);
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      s[(threadIdx.x >> 6) * 2] = a;
      s[(threadIdx.x >> 6) * 2 + 1] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      a += s[i * 2];
      b += s[i * 2 + 1];
    }
  }
}

template <typename T, typename W, int NE, int NT, int E>
__global__ __launch_bounds__(kThreads) void norm_forward_kernel(NormFwd a) {
  __shared__ float s_sum[kWaves];
  const int t = threadIdx.x % NT;
  constexpr int kRows = kThreads / NT;  // rows of a work-group at a time
  const int n = a.n;
  const float inv = 1.f / (float)n;
  float w[NE], b[NE];
  load_row<W, NE, NT, E>((const W*)a.w, n, t, w);
  if (a.b) {
    load_row<W, NE, NT, E>((const W*)a.b, n, t, b);
  } else {
#pragma unroll
    for (int e = 0; e < NE; ++e) b[e] = 0.f;
  }
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / NT; row < a.rows;
       row += (int64_t)gridDim.x * kRows) {
    float v[NE];
    load_row<T, NE, NT, E>((const T*)a.x + row * a.x_stride, n, t, v);
    if (a.residual) {
      float r[NE];
      load_row<T, NE, NT, E>((const T*)a.residual + row * a.r_stride, n, t, r);
      // the sum is rounded to the activations' type: the backward pass and the next
      // layer read it in that type, and the norm is of what they read
#pragma unroll
      for (int e = 0; e < NE; ++e) v[e] = (float)(T)(v[e] + r[e]);
      store_row<T, NE, NT, E>((T*)a.h + row * n, n, t, v);
    }
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) sum += v[e];
    const float mean = row_sum<NT>(sum, s_sum) * inv;
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      v[e] = column<NT, E>(e, t) < n ? v[e] - mean : 0.f;
      sq += v[e] * v[e];
    }
    const float rstd = 1.f / sqrtf(row_sum<NT>(sq, s_sum) * inv + a.eps);
#pragma unroll
    for (int e = 0; e < NE; ++e) v[e] = v[e] * rstd * w[e] + b[e];
    store_row<T, NE, NT, E>((T*)a.y + row * n, n, t, v);
    if (t == 0 && a.mean) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
  }
}

template <typename T, typename W, int NE, int NT, int E>
__global__ __launch_bounds__(kThreads) void norm_backward_kernel(NormBwd a) {
  __shared__ float s_sum[2 * kWaves];
  // one wave's columns at a time go through LDS to the work-group's sum
  __shared__ float s_cols[NT <= 64 ? kWaves * 64 * 4 : 1];
  const int t = threadIdx.x % NT;
  constexpr int kRows = kThreads / NT;
  const int n = a.n;
  const float inv = 1.f / (float)n;
  float w[NE], dw[NE], db[NE];
  load_row<W, NE, NT, E>((const W*)a.w, n, t, w);
#pragma unroll
  for (int e = 0; e < NE; ++e) dw[e] = db[e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / NT;
  RawRow<T, NE, NT, E> next_h, next_dy;
  float next_mean = 0.f, next_rstd = 0.f;
  auto fetch = [&](int64_t r) {
    next_h.load((const T*)a.h + r * a.h_stride, n, t);
    next_dy.load((const T*)a.dy + r * a.dy_stride, n, t);
    next_mean = a.mean[r];
    next_rstd = a.rstd[r];
  };
  if (row < a.rows) fetch(row);
  for (; row < a.rows; row += step) {
    float u[NE], g[NE];
    next_h.get(n, t, u);
    next_dy.get(n, t, g);
    const float mean = next_mean, rstd = next_rstd;
    if (row + step < a.rows) fetch(row + step);
    float sg = 0.f, sgu = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      u[e] = column<NT, E>(e, t) < n ? (u[e] - mean) * rstd : 0.f;
      dw[e] += g[e] * u[e];
      db[e] += g[e];
      g[e] *= w[e];
      sg += g[e];
      sgu += g[e] * u[e];
    }
    row_sum2<NT>(sg, sgu, s_sum);
    sg *= inv;
    sgu *= inv;
#pragma unroll
    for (int e = 0; e < NE; ++e) g[e] = rstd * (g[e] - sg - u[e] * sgu);
    if (a.dh) {
      load_row<T, NE, NT, E>((const T*)a.dh + row * n, n, t, u);
#pragma unroll
      for (int e = 0; e < NE; ++e) g[e] += u[e];
    }
    store_row<T, NE, NT, E>((T*)a.dx + row * n, n, t, g);
  }
  if (!a.dw && !a.db) return;
  if constexpr (NT <= 64) {
    // the rows that share a wave, then the waves in order, 4 of a thread's columns at a time
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      float(&x)[NE] = part ? db : dw;
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int o = 32; o >= NT; o >>= 1) x[e] += __shfl_xor(x[e], o);
#pragma unroll
      for (int c = 0; c < NE; c += 4) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) s_cols[(wave * 4 + j) * 64 + lane] = x[c + j];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float v = 0.f;
#pragma unroll
            for (int q = 0; q < kWaves; ++q) v += s_cols[(q * 4 + j) * 64 + lane];
            x[c + j] = v;
          }
        }
      }
    }
    if (threadIdx.x >= NT) return;
  }
  if (a.part) {
    float* p = a.part + (int64_t)blockIdx.x * 2 * n;
    store_row<float, NE, NT, E>(p, n, t, dw);
    store_row<float, NE, NT, E>(p + n, n, t, db);
  } else {
    if (a.dw) store_row<W, NE, NT, E>((W*)a.dw, n, t, dw);
    if (a.db) store_row<W, NE, NT, E>((W*)a.db, n, t, db);
  }
}

// Rows too long for the registers: a work-group a row, the row read once a step.  4,096 x
// 16,384 bf16 119 us, 2.3 TB/s counting each value once; what bounds it was not looked into, its
// moves are of one value.
template <typename T, typename W>
__global__ __launch_bounds__(kBigThreads) void norm_forward_big_kernel(NormFwd a) {
  __shared__ float s_sum[kBigThreads / 64];
  const int t = threadIdx.x, n = a.n;
  const float inv = 1.f / (float)n;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* h = (const T*)a.x + row * a.x_stride;
    float sum = 0.f;
    if (a.residual) {
      const T* x = h;
      const T* r = (const T*)a.residual + row * a.r_stride;
      T* to = (T*)a.h + row * n;
      for (int c = t; c < n; c += kBigThreads) {
        const T v = (T)((float)x[c] + (float)r[c]);
        to[c] = v;  // read again below by this thread alone
        sum += (float)v;
      }
      h = to;
    } else {
      for (int c = t; c < n; c += kBigThreads) sum += (float)h[c];
    }
    const float mean = row_sum<kBigThreads>(sum, s_sum) * inv;
    float sq = 0.f;
    for (int c = t; c < n; c += kBigThreads) {
      const float d = (float)h[c] - mean;
      sq += d * d;
    }
    const float rstd = 1.f / sqrtf(row_sum<kBigThreads>(sq, s_sum) * inv + a.eps);
    T* y = (T*)a.y + row * n;
    for (int c = t; c < n; c += kBigThreads)
      y[c] = (T)(((float)h[c] - mean) * rstd * (float)((const W*)a.w)[c] +
                 (a.b ? (float)((const W*)a.b)[c] : 0.f));
    if (t == 0 && a.mean) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
  }
}

// As above; the columns' sums stay in the work-group's partial row, which a thread
// reads and writes at its own columns only.  4,096 x 16,384 bf16: 359 us, 1.1 TB/s counting each
// value once.
template <typename T, typename W>
__global__ __launch_bounds__(kBigThreads) void norm_backward_big_kernel(NormBwd a) {
  __shared__ float s_sum[2 * kBigThreads / 64];
  const int t = threadIdx.x, n = a.n;
  const float inv = 1.f / (float)n;
  float* part = a.part + (int64_t)blockIdx.x * 2 * n;
  for (int c = t; c < 2 * n; c += kBigThreads) part[c] = 0.f;
  __syncthreads();
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* h = (const T*)a.h + row * a.h_stride;
    const T* dy = (const T*)a.dy + row * a.dy_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sg = 0.f, sgu = 0.f;
    for (int c = t; c < n; c += kBigThreads) {
      const float u = ((float)h[c] - mean) * rstd, d = (float)dy[c];
      const float g = d * (float)((const W*)a.w)[c];
      part[c] += d * u;
      part[n + c] += d;
      sg += g;
      sgu += g * u;
    }
    row_sum2<kBigThreads>(sg, sgu, s_sum);
    sg *= inv;
    sgu *= inv;
    T* dx = (T*)a.dx + row * n;
    const T* dh = a.dh ? (const T*)a.dh + row * n : nullptr;
    for (int c = t; c < n; c += kBigThreads) {
      const float u = ((float)h[c] - mean) * rstd;
      const float g = (float)dy[c] * (float)((const W*)a.w)[c];
      dx[c] = (T)(rstd * (g - sg - u * sgu) + (dh ? (float)dh[c] : 0.f));
    }
  }
}

// Adds the partial rows: a work-group takes 32 of the 2 n columns, its 32 groups of 32
// threads every 32nd row each, and LDS adds the groups in order.  Latency: 512 rows of 1,024
// columns 5 us.
template <typename W>
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ part,
                                                           int parts, int n, W* dw, W* db) {
  __shared__ float s[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + c;
  float v = 0.f;
  if (col < 2 * n) {
#pragma unroll 8
    for (int p = g; p < parts; p += 32) v += part[(int64_t)p * 2 * n + col];
  }
  s[g][c] = v;
  __syncthreads();
  if (g == 0 && col < 2 * n) {
    v = 0.f;
    for (int i = 0; i < 32; ++i) v += s[i][c];
    if (col < n) {
      if (dw) dw[col] = (W)v;
    } else if (db) {
      db[col - n] = (W)v;
    }
  }
}

// How a row is spread: NE values a thread (in moves of E, or 0), NT threads.  The smallest
// that holds it; 768 values, which moves of 8 would fill to three quarters, in moves of 4.
// 65,536 x 768 f16, forward and backward: 44 and 61 us, as a row of 1,024 47 and 79.
// 262,144 x 128 f16: 26 and 39 us, with 64 threads a row 64 and 145.
// f(NE, NT, E of an aligned row) as constants; false for rows that are too long.
template <int N>
using Int = std::integral_constant<int, N>;
template <typename F>
bool by_length(int n, F f) {
  if (n <= 128) f(Int<8>{}, Int<16>{}, Int<8>{});
  else if (n <= 512) f(Int<8>{}, Int<64>{}, Int<8>{});
  else if (n <= 768) f(Int<12>{}, Int<64>{}, Int<4>{});
  else if (n <= 1024) f(Int<16>{}, Int<64>{}, Int<8>{});
  else if (n <= 1536) f(Int<24>{}, Int<64>{}, Int<8>{});
  else if (n <= 2048) f(Int<32>{}, Int<64>{}, Int<8>{});
  else if (n <= 4096) f(Int<16>{}, Int<256>{}, Int<8>{});
  else if (n <= kMaxHeld) f(Int<32>{}, Int<256>{}, Int<8>{});
  else return false;
  return true;
}

// Work-groups of the backward pass.
int backward_groups(int64_t rows, int n) {
  int at_a_time = 1;  // rows of a work-group
  by_length(n, [&](auto, auto nt, auto) { at_a_time = kThreads / nt; });
  const int64_t steps = (rows + at_a_time - 1) / at_a_time;
  return (int)(steps < kMaxParts ? (steps > 0 ? steps : 1) : kMaxParts);
}

template <typename T, typename W>
void forward_typed(const NormFwd& a, bool vec, hipStream_t s) {
  const bool held = by_length(a.n, [&](auto ne, auto nt, auto e) {
    constexpr int kNE = decltype(ne)::value, kNT = decltype(nt)::value, kE = decltype(e)::value;
    constexpr int kRows = kThreads / kNT;
    const int64_t want = (a.rows + kRows - 1) / kRows;
    const int grid = (int)(want < 8192 ? want : 8192);
    if (vec) norm_forward_kernel<T, W, kNE, kNT, kE><<<grid, kThreads, 0, s>>>(a);
    else norm_forward_kernel<T, W, kNE, kNT, 0><<<grid, kThreads, 0, s>>>(a);
  });
  if (!held) {
    const int grid = (int)(a.rows < 4096 ? a.rows : 4096);
    norm_forward_big_kernel<T, W><<<grid, kBigThreads, 0, s>>>(a);
  }
}

template <typename T, typename W>
void backward_typed(const NormBwd& a, bool vec, int groups, hipStream_t s) {
  const int n = a.n;
  const bool held = by_length(n, [&](auto ne, auto nt, auto e) {
    constexpr int kNE = decltype(ne)::value, kNT = decltype(nt)::value, kE = decltype(e)::value;
    if (vec) norm_backward_kernel<T, W, kNE, kNT, kE><<<groups, kThreads, 0, s>>>(a);
    else norm_backward_kernel<T, W, kNE, kNT, 0><<<groups, kThreads, 0, s>>>(a);
  });
  if (!held) norm_backward_big_kernel<T, W><<<groups, kBigThreads, 0, s>>>(a);
  if (a.part && (a.dw || a.db))
    norm_reduce_kernel<W><<<(2 * n + 31) / 32, 1024, 0, s>>>(a.part, groups, n, (W*)a.dw,
                                                             (W*)a.db);
}

int check_norm(int32_t dtype, int32_t wdtype, int64_t rows, int32_t n) {
  if (!enc_dtype_ok(dtype))
    return set_error(SIEVE_EINVAL, "dtype = %d is not one of SIEVE_F32, SIEVE_F16, SIEVE_BF16",
                     dtype);
  if (wdtype != dtype && wdtype != SIEVE_F32)
    return set_error(SIEVE_EINVAL, "wdtype = %d must be dtype or SIEVE_F32", wdtype);
  if (rows < 0) return set_error(SIEVE_EINVAL, "rows is negative");
  if (n < 1) return set_error(SIEVE_EINVAL, "n = %d must be >= 1", n);
  if (n > kMaxN) return set_error(SIEVE_EUNSUPPORTED, "n = %d is above %d", n, kMaxN);
  return SIEVE_OK;
}

bool vec_ok(const void* p, int64_t stride, int size) {
  return ((uintptr_t)p & 15) == 0 && (stride * size & 15) == 0;
}

template <typename F>
void by_type(int32_t dtype, int32_t wdtype, F f) {
  if (dtype == SIEVE_F32) f(float{}, float{});
  else if (dtype == SIEVE_F16 && wdtype == SIEVE_F16) f(f16{}, f16{});
  else if (dtype == SIEVE_F16) f(f16{}, float{});
  else if (wdtype == SIEVE_BF16) f(bf16{}, bf16{});
  else f(bf16{}, float{});
}

}  // namespace

SIEVE_API int sieve_norm_forward(const void* x, int64_t x_stride, const void* residual,
                                 int64_t residual_stride, const void* weight, const void* bias,
                                 int32_t dtype, int32_t wdtype, int64_t rows, int32_t n, float eps,
                                 void* y, void* h, float* mean, float* rstd, void* stream) {
  clear_error();
  if (int st = check_norm(dtype, wdtype, rows, n)) return st;
  if (!(eps >= 0.f)) return set_error(SIEVE_EINVAL, "eps must be >= 0");
  if (rows == 0) return SIEVE_OK;
  if (!x || !weight || !y) return set_error(SIEVE_EINVAL, "x, weight and y must be non-NULL");
  if ((residual != nullptr) != (h != nullptr))
    return set_error(SIEVE_EINVAL, "h is given with a residual, and only then");
  if ((mean != nullptr) != (rstd != nullptr))
    return set_error(SIEVE_EINVAL, "mean and rstd are given together");
  if (x_stride < n || (residual && residual_stride < n))
    return set_error(SIEVE_EINVAL, "a row stride is below n = %d", n);
  if (h && h == y) return set_error(SIEVE_EINVAL, "y and h are the same buffer");
  const int sz = enc_size(dtype), wsz = enc_size(wdtype);
  const bool vec = n % 8 == 0 && vec_ok(x, x_stride, sz) && vec_ok(y, n, sz) &&
                   vec_ok(weight, n, wsz) && (!bias || vec_ok(bias, n, wsz)) &&
                   (!residual || (vec_ok(residual, residual_stride, sz) && vec_ok(h, n, sz)));
  const NormFwd a{x, residual, weight, bias, x_stride, residual_stride, rows, n, eps,
                  y, h, mean, rstd};
  by_type(dtype, wdtype, [&](auto t, auto w) {
    forward_typed<decltype(t), decltype(w)>(a, vec, (hipStream_t)stream);
  });
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}

SIEVE_API int64_t sieve_norm_workspace(int64_t rows, int32_t n) {
  clear_error();
  if (int st = check_norm(SIEVE_F32, SIEVE_F32, rows, n)) return st;
  const int groups = backward_groups(rows, n);
  return groups == 1 && n <= kMaxHeld ? 0 : (int64_t)groups * 2 * n * (int64_t)sizeof(float);
}

SIEVE_API int sieve_norm_backward(const void* dy, int64_t dy_stride, const void* h,
                                  int64_t h_stride, const void* weight, const float* mean,
                                  const float* rstd, const void* dh, int32_t dtype,
                                  int32_t wdtype, int64_t rows, int32_t n, void* dx, void* dweight,
                                  void* dbias, void* workspace, int64_t workspace_bytes,
                                  void* stream) {
  clear_error();
  if (int st = check_norm(dtype, wdtype, rows, n)) return st;
  if (!weight) return set_error(SIEVE_EINVAL, "weight must be non-NULL");
  if (rows > 0 && (!dy || !h || !mean || !rstd || !dx))
    return set_error(SIEVE_EINVAL, "dy, h, mean, rstd and dx must be non-NULL when rows > 0");
  if (rows > 0 && (dy_stride < n || h_stride < n))
    return set_error(SIEVE_EINVAL, "a row stride is below n = %d", n);
  const int64_t need = sieve_norm_workspace(rows, n);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
    return set_error(SIEVE_EINVAL, "workspace must be 16-byte aligned and hold %lld bytes",
                     (long long)need);
  const int sz = enc_size(dtype), wsz = enc_size(wdtype);
  const bool vec = n % 8 == 0 && vec_ok(dy, dy_stride, sz) && vec_ok(h, h_stride, sz) &&
                   vec_ok(weight, n, wsz) && vec_ok(dx, n, sz) && vec_ok(dweight, n, wsz) &&
                   vec_ok(dbias, n, wsz) && (!dh || vec_ok(dh, n, sz));
  const NormBwd a{dy, h, weight, dh, mean, rstd, dy_stride, h_stride, rows, n, dx, dweight, dbias,
                  need > 0 ? (float*)workspace : nullptr};
  const int groups = backward_groups(rows, n);
  by_type(dtype, wdtype, [&](auto t, auto w) {
    backward_typed<decltype(t), decltype(w)>(a, vec, groups, (hipStream_t)stream);
  });
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}
