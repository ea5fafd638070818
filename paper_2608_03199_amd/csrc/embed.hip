// embed.hip -- rows of a table by token number, and the table's gradient.
//
//   out[t] = scale table[ids[t]]             (zeros where ids[t] is not in [0, vocab))
//   dtable[v] = scale sum over t with ids[t] = v of dy[t]   (+ dtable[v])
//
// Both are bound by memory: the forward pass reads a row and writes one, the backward pass
// reads dy once and writes the table's gradient once, if what it reads of a row is summed in
// registers.  So the tokens are sorted by their numbers first, and a row's tokens are then next
// to each other.
//
// The sort is a stable radix sort of (number, token) pairs, so equal tokens stay in the order of
// the batch: a tile's digits are counted, the counts summed over the tiles, and each pair is
// written to its place.  Digits are of up to 11 bits: one pass for vocabularies below 2^11, two
// below 2^22.  Sums are in a fixed order, without atomics: equal calls give equal bits.
//
// A frequent token would leave one row with most of the work, so runs of equal numbers are
// summed ahead in pieces: a piece of 32 sorted places that holds one number alone is summed by
// itself, so is a piece of 32 such pieces, and so on.  A row then adds up to 62 of each kind.
//
// A row moves 16 bytes a thread, wherever it lies.  Measured: 262,144 rows of 768 f16 are written
// in 117 us, 3.9 TB/s.  65,536 x 1,024 bf16 of a table of 50,000 fp32 rows: forward 49 us; backward
// 15 us a pass of the sort, 16 for the runs and 85 for the rows, of which what they read
// and write, 339 MB, takes 69 at the rate of a copy.
#include <algorithm>

#include "enc_common.h"

using namespace sieve;

namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kThreads = 256;
constexpr int kMaxN = 65536;
constexpr int64_t kMaxCount = 0x7fffffff;
constexpr int64_t kMaxVocab = 0x7ffffffe;

// ---- forward ---------------------------------------------------------------------------------

struct EmbedFwd {
  const void *ids, *table;
  int64_t count, t_stride, vocab;
  int n;
  float scale;
  void* out;
  int rows;              // rows of a work-group
  int pieces;            // moves of a row
  uint32_t mul, shift;   // index / pieces = (index * mul) >> shift
};

// E values of type T as floats, in one move.  kWhole: they lie at a multiple of 16 bytes (or of
// E values' size); else anywhere, and only `left` of them are there.
template <typename T, int E, bool kWhole>
__device__ __forceinline__ void load_values(const T* p, int left, float (&v)[E]) {
  if constexpr (kWhole) {
    const EncVec<T, E> q = enc_load<T, E>(p);
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = (float)q.v[j];
  } else if (left >= E) {
    T q[E];
    __builtin_memcpy(q, p, sizeof(q));
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = (float)q[j];
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = j < left ? (float)p[j] : 0.f;
  }
}
template <typename T, int E, bool kWhole>
__device__ __forceinline__ void store_values(T* p, int left, const float (&v)[E]) {
  if constexpr (kWhole) {
    EncVec<T, E> q;
#pragma unroll
    for (int j = 0; j < E; ++j) q.v[j] = (T)v[j];
    enc_store<T, E>(p, q);
  } else if (left >= E) {
    T q[E];
#pragma unroll
    for (int j = 0; j < E; ++j) q[j] = (T)v[j];
    __builtin_memcpy(p, q, sizeof(q));
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (j < left) p[j] = (T)v[j];
  }
}

constexpr int kMoves = 4;

template <typename W, typename T, typename I, int E, bool kWhole>
__global__ __launch_bounds__(kThreads) void embed_forward_kernel(EmbedFwd a) {
  for (int64_t first = (int64_t)blockIdx.x * a.rows; first < a.count;
       first += (int64_t)gridDim.x * a.rows) {
    const int64_t left = a.count - first;
    const int rows = left < a.rows ? (int)left : a.rows;
    const I* ids = (const I*)a.ids + first;
    T* out = (T*)a.out + first * a.n;
    const int all = rows * a.pieces;
    // kMoves of a thread at a time: their numbers, then their values are on the way together
    for (int i0 = threadIdx.x; i0 < all; i0 += kMoves * kThreads) {
      int64_t id[kMoves];
      int row[kMoves];
#pragma unroll
      for (int u = 0; u < kMoves; ++u) {
        const int i = i0 + u * kThreads;
        row[u] = (int)(((uint64_t)(uint32_t)i * a.mul) >> a.shift);
        id[u] = i < all ? (int64_t)ids[row[u]] : -1;
      }
      float v[kMoves][E];
#pragma unroll
      for (int u = 0; u < kMoves; ++u) {
        const int col = (i0 + u * kThreads - row[u] * a.pieces) * E;
        if (id[u] >= 0 && id[u] < a.vocab) {
          load_values<W, E, kWhole>((const W*)a.table + id[u] * a.t_stride + col, a.n - col, v[u]);
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) v[u][j] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < kMoves; ++u) {
        const int i = i0 + u * kThreads, col = (i - row[u] * a.pieces) * E;
#pragma unroll
        for (int j = 0; j < E; ++j) v[u][j] *= a.scale;
        if (i < all) store_values<T, E, kWhole>(out + (int64_t)row[u] * a.n + col, a.n - col, v[u]);
      }
    }
  }
}

// ---- sorting ---------------------------------------------------------------------------------

constexpr int kMaxDigit = 11;                 // bits of a digit
constexpr int kBins = 1 << kMaxDigit;
constexpr int kRounds = 8;                    // pairs of a thread
constexpr int kTile = kThreads * kRounds;     // pairs of a work-group
constexpr int kWaves = kThreads / 64;
constexpr int kEach = kBins / kThreads;       // bins of a thread
// Up to so many counts a thread every tile adds them up by itself; more go through a kernel of
// their own, another launch.  65,536 tokens, 8,000 rows, 32 counts a thread: 54 us for 60 with the
// kernel; 20,001 tokens, 2,000 rows, 80: 59 us without it for 43.
constexpr int kFewCounts = 64;
inline __host__ __device__ bool few_counts(int tiles, int bins) {
  return tiles * ((bins + kThreads - 1) / kThreads) <= kFewCounts;
}

struct Pass {
  const void* ids;                // the first pass reads these (I), later ones `from`
  const uint32_t *from_key, *from_at;
  uint32_t *to_key, *to_at;
  uint32_t* counts;               // [tiles][bins], then their exclusive sums along the tiles
  uint32_t* totals;               // [bins]
  int64_t count, vocab;
  int tiles, shift, bits;
};

// A token's sort key: its number, or vocab where that is not in the table.
template <typename I, bool kFirst>
__device__ __forceinline__ uint32_t key_of(const Pass& a, int64_t i) {
  if constexpr (kFirst) {
    const int64_t id = (int64_t)((const I*)a.ids)[i];
    return (uint32_t)(id >= 0 && id < a.vocab ? id : a.vocab);
  } else {
    return a.from_key[i];
  }
}

template <typename I, bool kFirst>
__global__ __launch_bounds__(kThreads) void sort_count_kernel(Pass a) {
  __shared__ uint32_t s_count[kBins];
  const int bins = 1 << a.bits;
  for (int b = threadIdx.x; b < bins; b += kThreads) s_count[b] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = (int64_t)blockIdx.x * kTile + r * kThreads + threadIdx.x;
    if (i < a.count)
      atomicAdd(&s_count[(key_of<I, kFirst>(a, i) >> a.shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kThreads)
    a.counts[(int64_t)blockIdx.x * bins + b] = s_count[b];
}

// A work-group sums 32 digits' counts along the tiles, in 8 runs of tiles.
__global__ __launch_bounds__(kThreads) void sort_sum_kernel(Pass a) {
  __shared__ uint32_t s_run[8][32];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, bins = 1 << a.bits;
  const int bin = blockIdx.x * 32 + c, per = (a.tiles + 7) / 8;
  const int first = g * per, last = first + per < a.tiles ? first + per : a.tiles;
  uint32_t sum = 0;
  if (bin < bins) {
#pragma unroll 8
    for (int t = first; t < last; ++t) sum += a.counts[(int64_t)t * bins + bin];
  }
  s_run[g][c] = sum;
  __syncthreads();
  if (bin >= bins) return;
  uint32_t before = 0;
  for (int i = 0; i < g; ++i) before += s_run[i][c];
#pragma unroll 8
  for (int t = first; t < last; ++t) {
    const uint32_t own = a.counts[(int64_t)t * bins + bin];
    a.counts[(int64_t)t * bins + bin] = before;
    before += own;
  }
  if (g == 7) a.totals[bin] = before;
}

// Exclusive sums of `bins` values in LDS, by the whole work-group.
__device__ __forceinline__ void sum_bins(uint32_t* s, int bins, uint32_t* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int each = (bins + kThreads - 1) / kThreads, first = threadIdx.x * each;
  uint32_t sum = 0;
  for (int j = 0; j < each; ++j) sum += first + j < bins ? s[first + j] : 0;
  uint32_t all = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(all, o);
    if (lane >= o) all += up;
  }
  if (lane == 63) s_wave[wave] = all;
  __syncthreads();
  uint32_t before = all - sum;
  for (int w = 0; w < wave; ++w) before += s_wave[w];
  for (int j = 0; j < each; ++j)
    if (first + j < bins) {
      const uint32_t own = s[first + j];
      s[first + j] = before;
      before += own;
    }
  __syncthreads();
}

// Orders a wave's own LDS reads and writes.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Writes a tile's pairs to their places.  A wave takes the tile's pairs 512 w .. 512 w + 511 in
// order, 64 at a time: a pair's rank among the equal digits of its 64 comes from ballots.
template <typename I, bool kFirst>
__global__ __launch_bounds__(kThreads) void sort_place_kernel(Pass a) {
  __shared__ uint32_t s_wave[kWaves], s_total[kBins];
  __shared__ uint32_t s_count[kWaves][kBins];
  const int bins = 1 << a.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = (int64_t)blockIdx.x * kTile + wave * (kTile / kWaves);
  uint32_t key[kRounds], at[kRounds], rank[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = first + r * 64 + lane;
    key[r] = i < a.count ? key_of<I, kFirst>(a, i) : 0;
    at[r] = kFirst || i >= a.count ? (uint32_t)i : a.from_at[i];
  }
  // all pairs of each bin, and those of the tiles before: bins threadIdx.x + 256 j
  uint32_t before[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int b = threadIdx.x + j * kThreads;
    before[j] = 0;
    if (b >= bins) break;
    uint32_t total = 0;
    if (!few_counts(a.tiles, bins)) {
      total = a.totals[b];
      before[j] = a.counts[(int64_t)blockIdx.x * bins + b];
    } else if (a.tiles > 1) {
#pragma unroll 16
      for (int t = 0; t < a.tiles; ++t) {
        const uint32_t c = a.counts[(int64_t)t * bins + b];
        total += c;
        before[j] += t < (int)blockIdx.x ? c : 0;
      }
    }
    s_total[b] = total;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s_count[w][b] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const bool ok = first + r * 64 + lane < a.count;
    const uint32_t digit = (key[r] >> a.shift) & (bins - 1);
    uint64_t same = __ballot(ok);
    for (int b = 0; b < a.bits; ++b) {
      const uint64_t has = __ballot(digit >> b & 1);
      same &= (digit >> b & 1) ? has : ~has;
    }
    const uint64_t below = same & ((uint64_t(1) << lane) - 1);
    rank[r] = ok ? s_count[wave][digit] + (uint32_t)__popcll(below) : 0;
    wave_fence();
    if (ok && below == 0) s_count[wave][digit] += (uint32_t)__popcll(same);
    wave_fence();
  }
  __syncthreads();
  if (a.tiles == 1) {  // no counts: they are this tile's
    for (int b = threadIdx.x; b < bins; b += kThreads) {
      uint32_t total = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) total += s_count[w][b];
      s_total[b] = total;
    }
    __syncthreads();
  }
  sum_bins(s_total, bins, s_wave);
  // where the waves' pairs of each digit begin
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int b = threadIdx.x + j * kThreads;
    if (b >= bins) break;
    uint32_t to = s_total[b] + before[j];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = s_count[w][b];
      s_count[w][b] = to;
      to += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    if (first + r * 64 + lane >= a.count) continue;
    const uint32_t to = s_count[wave][(key[r] >> a.shift) & (bins - 1)] + rank[r];
    a.to_key[to] = key[r];
    a.to_at[to] = at[r];
  }
}

// ---- backward --------------------------------------------------------------------------------

// 65,536 x 1,024 bf16, 50,000 rows, the rows' kernel with four values ahead: 105 us; with runs of
// 64 it takes 124, with 16 it is 8% shorter but more kinds of pieces are launched; with 8 rows a
// work-group 125, with 4 148, with 32 no less.
constexpr int kRun = 32;       // places of a piece, pieces of a piece of the next kind
constexpr int kKinds = 6;      // of 32^kind places each; 32^7 are more than kMaxCount
constexpr int64_t places_of(int kind) { return kind ? kRun * places_of(kind - 1) : 1; }
static_assert(places_of(kKinds) <= kMaxCount && places_of(kKinds + 1) > kMaxCount);
constexpr int kMaxRows = 16;   // table rows of a work-group

struct EmbedBwd {
  const void* dy;
  int64_t dy_stride;
  const uint32_t *key, *at;    // sorted
  int64_t count, vocab;
  int n, pitch;                // pitch: values between partial sums
  float scale;
  int accumulate;
  void* dtable;
  float* part[kKinds + 1];     // part[k][j]: the sum of places 32^k j .. 32^k (j + 1) - 1
  int kinds;                   // kinds that fit into count
  int group;                   // threads of a row
  int rows;                    // table rows of a work-group
};

template <typename T, int E, bool kWhole>
struct Sum {
  const EmbedBwd& a;
  int col;
  float v[E];
  __device__ __forceinline__ Sum(const EmbedBwd& a_, int col_) : a(a_), col(col_) {
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = 0.f;
  }
  // Adds load(i) for i = 0 .. count - 1, in order, kAhead of them on their way at a time: 8 values
  // of 16 bits twice, 91 us where one takes 101 and four 105 (as above, with rows found by halves).
  static constexpr int kAhead = 16 / E;
  template <typename F>
  __device__ __forceinline__ void all(int count, F load) {
    for (int i = 0; i < count; i += kAhead) {
      float x[kAhead][E];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i + u < count) {
          load(i + u, x[u]);
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) x[u][j] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] += x[u][j];
    }
  }
  // Sorted places begin .. end - 1.  The row's threads (of a wave) load the tokens' numbers
  // together and pass them round: one wait for all of them.
  __device__ __forceinline__ void places(int64_t begin, int64_t end) {
    const int many = a.group < 64 ? a.group : 64, lane = threadIdx.x & 63;
    const int first = lane & ~(many - 1);
    for (int64_t p = begin; p < end; p += many) {
      const int count = end - p < many ? (int)(end - p) : many;
      const uint32_t mine = a.at[p + (lane - first < count ? lane - first : count - 1)];
      all(count, [&](int i, float (&x)[E]) {
        const int64_t token = (int64_t)(uint32_t)__shfl((int)mine, first + i);
        load_values<T, E, kWhole>((const T*)a.dy + token * a.dy_stride + col, a.n - col, x);
      });
    }
  }
  __device__ __forceinline__ void pieces(int kind, int64_t begin, int64_t end) {
    all((int)(end - begin), [&](int i, float (&x)[E]) {
      load_values<float, E, true>(a.part[kind] + (begin + i) * a.pitch + col, E, x);
    });
  }
  // places of one number: what is left at both ends of the largest pieces inside, kind by kind
  __device__ __forceinline__ void interval(int64_t begin, int64_t end) {
    for (int kind = 0;; ++kind) {
      const int64_t up = (begin + kRun - 1) / kRun, down = end / kRun;
      const bool last = kind == a.kinds || up >= down;
      const int64_t head = last ? end : up * kRun, tail = last ? end : down * kRun;
      if (kind == 0) {
        places(begin, head);
        places(tail, end);
      } else {
        pieces(kind, begin, head);
        pieces(kind, tail, end);
      }
      if (last) break;
      begin = up;
      end = down;
    }
  }
};

// Sums of the pieces of a kind that hold one number alone, by groups of threads.
template <typename T, int E, bool kWhole>
__global__ __launch_bounds__(kThreads) void embed_pieces_kernel(EmbedBwd a, int kind,
                                                                int64_t span) {
  const int lane = threadIdx.x % a.group;
  const int groups = kThreads / a.group;
  for (int64_t j = (int64_t)blockIdx.x * groups + threadIdx.x / a.group;
       (j + 1) * span <= a.count; j += (int64_t)gridDim.x * groups) {
    const uint32_t key = a.key[j * span];
    if (key != a.key[(j + 1) * span - 1] || key == (uint32_t)a.vocab) continue;
    for (int c = 0; c < a.n; c += a.group * E) {
      const int col = c + lane * E;
      Sum<T, E, kWhole> s(a, col < a.n ? col : 0);  // a row's threads stay together
      if (kind == 1) s.places(j * kRun, (j + 1) * kRun);
      else s.pieces(kind - 1, j * kRun, (j + 1) * kRun);
      if (col < a.n) store_values<float, E, true>(a.part[kind] + j * a.pitch + col, E, s.v);
    }
  }
}

template <typename T, typename W, int E, bool kWhole>
__global__ __launch_bounds__(kThreads) void embed_rows_kernel(EmbedBwd a) {
  __shared__ int64_t s_begin[kMaxRows + 1];
  const int lane = threadIdx.x % a.group;
  for (int64_t v0 = (int64_t)blockIdx.x * a.rows; v0 < a.vocab;
       v0 += (int64_t)gridDim.x * a.rows) {
    __syncthreads();  // the rows before have been read
    if (threadIdx.x < 8 * (a.rows + 1)) {
      // the first place whose number is not below v, which is one of lo .. hi: 8 threads look at 8
      // places at a time, of which the first c hold numbers below it: this kernel takes 20.8 us at
      // 20,001 x 515 fp32 and 85 at 65,536 x 1,024 bf16, by halves 23.6 and 91
      const int64_t v = v0 + threadIdx.x / 8;
      uint32_t lo = 0, hi = (uint32_t)a.count;
      while (lo < hi) {
        const uint32_t step = (hi - lo + 8) / 9, at = lo + (threadIdx.x % 8 + 1) * step - 1;
        const uint64_t below = __ballot(at < hi && (int64_t)a.key[at] < v);
        const uint32_t c = __popc((uint32_t)(below >> (threadIdx.x & 56)) & 255u);
        if (c < 8) hi = min(hi, lo + (c + 1) * step - 1);
        lo += c * step;
      }
      if (threadIdx.x % 8 == 0) s_begin[threadIdx.x / 8] = lo;
    }
    __syncthreads();
    for (int r = threadIdx.x / a.group; r < a.rows && v0 + r < a.vocab; r += kThreads / a.group) {
      const int64_t begin = s_begin[r], end = s_begin[r + 1];
      if (a.accumulate && begin == end) continue;
      W* row = (W*)a.dtable + (v0 + r) * a.n;
      for (int c = 0; c < a.n; c += a.group * E) {
        const int col = c + lane * E;
        Sum<T, E, kWhole> s(a, col < a.n ? col : 0);  // a row's threads stay together
        s.interval(begin, end);
        if (col >= a.n) continue;
#pragma unroll
        for (int j = 0; j < E; ++j) s.v[j] *= a.scale;
        if (a.accumulate) {
          float old[E];
          load_values<W, E, kWhole>(row + col, a.n - col, old);
#pragma unroll
          for (int j = 0; j < E; ++j) s.v[j] += old[j];
        }
        store_values<W, E, kWhole>(row + col, a.n - col, s.v);
      }
    }
  }
}

// ---- host ------------------------------------------------------------------------------------

int64_t round256(int64_t n) { return (n + 255) & ~int64_t(255); }

// Where a backward pass keeps what; offsets in bytes.
struct Layout {
  int tiles, passes, bits, kinds, pitch;
  int64_t key[2], at[2], counts, totals, part[kKinds + 1], bytes;
};

Layout layout_of(int64_t count, int64_t vocab, int32_t n) {
  Layout l{};
  int bits = 1;
  while (vocab >> bits) ++bits;  // keys go up to vocab
  l.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  l.bits = (bits + l.passes - 1) / l.passes;
  l.tiles = (int)((count + kTile - 1) / kTile);
  l.pitch = (n + 7) & ~7;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t was = at;
    at += round256(bytes);
    return was;
  };
  for (int i = 0; i < 2; ++i) {
    l.key[i] = take(count * 4);
    l.at[i] = take(count * 4);
  }
  l.counts = take(((int64_t)l.tiles << l.bits) * 4);
  l.totals = take(((int64_t)1 << l.bits) * 4);
  for (int64_t span = kRun; span <= count; span *= kRun)
    l.part[++l.kinds] = take(count / span * l.pitch * 4);
  l.bytes = at;
  return l;
}

int check_embed(int32_t dtype, int32_t tdtype, int32_t id_bytes, int64_t count, int64_t vocab,
                int32_t n) {
  if (!enc_dtype_ok(dtype))
    return set_error(SIEVE_EINVAL, "dtype = %d is not one of SIEVE_F32, SIEVE_F16, SIEVE_BF16",
                     dtype);
  if (tdtype != dtype && tdtype != SIEVE_F32)
    return set_error(SIEVE_EINVAL, "tdtype = %d must be dtype or SIEVE_F32", tdtype);
  if (id_bytes != 4 && id_bytes != 8)
    return set_error(SIEVE_EINVAL, "id_bytes = %d must be 4 or 8", id_bytes);
  if (count < 0) return set_error(SIEVE_EINVAL, "count is negative");
  if (vocab < 1) return set_error(SIEVE_EINVAL, "vocab must be >= 1");
  if (n < 1) return set_error(SIEVE_EINVAL, "n = %d must be >= 1", n);
  if (n > kMaxN) return set_error(SIEVE_EUNSUPPORTED, "n = %d is above %d", n, kMaxN);
  if (count > kMaxCount)
    return set_error(SIEVE_EUNSUPPORTED, "count is above %lld", (long long)kMaxCount);
  if (vocab > kMaxVocab)
    return set_error(SIEVE_EUNSUPPORTED, "vocab is above %lld", (long long)kMaxVocab);
  return SIEVE_OK;
}

bool vec_ok(const void* p, int64_t stride, int size) {
  return ((uintptr_t)p & 15) == 0 && (stride * size & 15) == 0;
}

// f(values' type, table's type)
template <typename F>
void by_type(int32_t dtype, int32_t tdtype, F f) {
  if (dtype == SIEVE_F32) f(float{}, float{});
  else if (dtype == SIEVE_F16 && tdtype == SIEVE_F16) f(f16{}, f16{});
  else if (dtype == SIEVE_F16) f(f16{}, float{});
  else if (tdtype == SIEVE_BF16) f(bf16{}, bf16{});
  else f(bf16{}, float{});
}

// Work-groups for so many pieces of work; the kernels take what is left in turns.
int grid_of(int64_t work) { return (int)(work < (1 << 20) ? work : 1 << 20); }

template <typename I>
void sort(Pass a, const Layout& l, char* w, hipStream_t s) {
  const int bins = 1 << l.bits;
  a.bits = l.bits;
  a.tiles = l.tiles;
  a.counts = (uint32_t*)(w + l.counts);
  a.totals = (uint32_t*)(w + l.totals);
  for (int p = 0; p < l.passes; ++p) {
    a.shift = p * l.bits;
    a.from_key = (const uint32_t*)(w + l.key[(p + 1) & 1]);
    a.from_at = (const uint32_t*)(w + l.at[(p + 1) & 1]);
    a.to_key = (uint32_t*)(w + l.key[p & 1]);
    a.to_at = (uint32_t*)(w + l.at[p & 1]);
    if (l.tiles > 1) {
      if (p == 0) sort_count_kernel<I, true><<<l.tiles, kThreads, 0, s>>>(a);
      else sort_count_kernel<I, false><<<l.tiles, kThreads, 0, s>>>(a);
    }
    if (!few_counts(l.tiles, bins)) sort_sum_kernel<<<(bins + 31) / 32, kThreads, 0, s>>>(a);
    if (p == 0) sort_place_kernel<I, true><<<l.tiles, kThreads, 0, s>>>(a);
    else sort_place_kernel<I, false><<<l.tiles, kThreads, 0, s>>>(a);
  }
}

template <typename T, typename W, int E, bool kWhole>
void backward_typed(EmbedBwd a, hipStream_t s) {
  const int pieces = (a.n + E - 1) / E;
  a.group = 8;
  while (a.group < pieces && a.group < kThreads) a.group *= 2;
  const int groups = kThreads / a.group;
  int64_t span = 1;
  for (int kind = 1; kind <= a.kinds; ++kind) {
    span *= kRun;
    const int grid = grid_of((a.count / span + groups - 1) / groups);
    embed_pieces_kernel<T, E, kWhole><<<grid, kThreads, 0, s>>>(a, kind, span);
  }
  // few in a small table, 2,000 x 515 fp32: 43 us for 81 with 16; but one a group of threads,
  // 65,536 tokens of 8,000 x 256 bf16: 45 us for 54 with 3 rows, which leave half of them idle
  const int64_t want = std::max<int64_t>(a.vocab / 2048, groups);
  a.rows = (int)std::min<int64_t>(want, kMaxRows);
  const int grid = grid_of((a.vocab + a.rows - 1) / a.rows);
  embed_rows_kernel<T, W, E, kWhole><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

SIEVE_API int sieve_embed_forward(const void* ids, int32_t id_bytes, int64_t count,
                                  const void* table, int64_t table_stride, int32_t tdtype,
                                  int64_t vocab, int32_t n, float scale, void* out, int32_t dtype,
                                  void* stream) {
  clear_error();
  if (int st = check_embed(dtype, tdtype, id_bytes, count, vocab, n)) return st;
  if (count == 0) return SIEVE_OK;
  if (!ids || !table || !out) return set_error(SIEVE_EINVAL, "ids, table and out must be non-NULL");
  if (table_stride < n) return set_error(SIEVE_EINVAL, "table_stride is below n = %d", n);
  by_type(dtype, tdtype, [&](auto t, auto w) {
    typedef decltype(t) T;
    typedef decltype(w) W;
    constexpr int kE = 16 / (int)sizeof(T);
    const bool whole = n % kE == 0 && vec_ok(table, table_stride, sizeof(W)) &&
                       vec_ok(out, n, sizeof(T));
    EmbedFwd a{ids, table, count, table_stride, vocab, n, scale, out, 0, 0, 0, 0};
    a.pieces = (n + kE - 1) / kE;
    // kMoves a thread; few rows where there are few
    a.rows = 4 * kThreads / a.pieces;
    while (a.rows > 1 && count / a.rows < 512) a.rows /= 2;
    if (a.rows < 1) a.rows = 1;
    // indexes stay below 2^17: exact with a multiplier of 2^36 / pieces rounded up
    a.shift = 36;
    a.mul = (uint32_t)(((uint64_t(1) << 36) + a.pieces - 1) / a.pieces);
    if (a.pieces < 32) {
      a.shift = 31;
      a.mul = (uint32_t)(((uint64_t(1) << 31) + a.pieces - 1) / a.pieces);
    }
    const int grid = grid_of((count + a.rows - 1) / a.rows);
    hipStream_t s = (hipStream_t)stream;
    if (id_bytes == 8) {
      if (whole) embed_forward_kernel<W, T, int64_t, kE, true><<<grid, kThreads, 0, s>>>(a);
      else embed_forward_kernel<W, T, int64_t, kE, false><<<grid, kThreads, 0, s>>>(a);
    } else {
      if (whole) embed_forward_kernel<W, T, int32_t, kE, true><<<grid, kThreads, 0, s>>>(a);
      else embed_forward_kernel<W, T, int32_t, kE, false><<<grid, kThreads, 0, s>>>(a);
    }
  });
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}

SIEVE_API int64_t sieve_embed_workspace(int64_t count, int64_t vocab, int32_t n) {
  clear_error();
  if (int st = check_embed(SIEVE_F32, SIEVE_F32, 8, count, vocab, n)) return st;
  return count ? layout_of(count, vocab, n).bytes : 0;
}

SIEVE_API int sieve_embed_backward(const void* dy, int64_t dy_stride, int32_t dtype,
                                   const void* ids, int32_t id_bytes, int64_t count, int64_t vocab,
                                   int32_t n, float scale, int32_t accumulate, void* dtable,
                                   int32_t tdtype, void* workspace, int64_t workspace_bytes,
                                   void* stream) {
  clear_error();
  if (int st = check_embed(dtype, tdtype, id_bytes, count, vocab, n)) return st;
  if (accumulate != 0 && accumulate != 1)
    return set_error(SIEVE_EINVAL, "accumulate must be 0 or 1");
  if (!dtable) return set_error(SIEVE_EINVAL, "dtable must be non-NULL");
  if (count > 0 && (!dy || !ids))
    return set_error(SIEVE_EINVAL, "dy and ids must be non-NULL when count > 0");
  if (count > 0 && dy_stride < n) return set_error(SIEVE_EINVAL, "dy_stride is below n = %d", n);
  const Layout l = layout_of(count, vocab, n);
  if (count > 0 && (!workspace || workspace_bytes < l.bytes || ((uintptr_t)workspace & 15)))
    return set_error(SIEVE_EINVAL, "workspace must be 16-byte aligned and hold %lld bytes",
                     (long long)l.bytes);
  if (count == 0 && accumulate) return SIEVE_OK;
  char* w = (char*)workspace;
  hipStream_t s = (hipStream_t)stream;
  EmbedBwd a{};
  if (count > 0) {
    Pass p{};
    p.ids = ids;
    p.count = count;
    p.vocab = vocab;
    if (id_bytes == 8) sort<int64_t>(p, l, w, s);
    else sort<int32_t>(p, l, w, s);
    const int last = (l.passes - 1) & 1;
    a.key = (const uint32_t*)(w + l.key[last]);
    a.at = (const uint32_t*)(w + l.at[last]);
    for (int k = 1; k <= l.kinds; ++k) a.part[k] = (float*)(w + l.part[k]);
  }
  a.dy = dy;
  a.dy_stride = dy_stride;
  a.count = count;
  a.vocab = vocab;
  a.n = n;
  a.pitch = l.pitch;
  a.scale = scale;
  a.accumulate = accumulate;
  a.dtable = dtable;
  a.kinds = l.kinds;
  by_type(dtype, tdtype, [&](auto t, auto wt) {
    typedef decltype(t) T;
    typedef decltype(wt) W;
    constexpr int kE = 16 / (int)sizeof(T);
    const bool whole = n % kE == 0 && (count == 0 || vec_ok(dy, dy_stride, sizeof(T))) &&
                       vec_ok(dtable, n, sizeof(W));
    if (whole) backward_typed<T, W, kE, true>(a, s);
    else backward_typed<T, W, kE, false>(a, s);
  });
  ENC_HIP_TRY(hipGetLastError());
  return SIEVE_OK;
}
