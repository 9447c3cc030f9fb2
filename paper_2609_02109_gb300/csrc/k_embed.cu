// Embedding lookup and the gradient of its table (the operators' section of include/mf.h).
//
// Forward: a row of the output is a row of the table, times a factor.  Bound by memory: a thread moves pieces of 16 bytes
// (where rows allow; else the widest that they do), several in flight.
//
// Backward: tokens are sorted by their row (a stable radix sort, so that equal rows keep the tokens' order), and each row's
// gradient is the sum of a run of sorted tokens.  A unit is a fixed number of sorted tokens; a thread adds up one piece of
// a row over a unit and writes a run's sum where the run ends, or, where a run passes the unit's border, a partial sum, and
// the partial sums of a row are added up in the order of the units.  No atomics on values: equal calls give equal bits.
// Rows that no token names are zeroed by blocks of the same launch, from a bitmap of the rows that are named.
//
// Measured, 65536 tokens of 1024 bf16 values over 100,003 rows (486 MB with the lookup, 72 us at the copy rate): 166 us a
// lookup and gradient.  Cold, by launches: lookup 43, four launches of the sort 39 (32 blocks: latency), the bitmap 4, sums
// and zeroed rows 52 (5.4 TB/s), joined runs 22.
#include <algorithm>

#include "mf_ops.cuh"

namespace mf {
namespace {

// V consecutive values of a row.
template <typename T, int V>
struct alignas(sizeof(T) * V) Piece {
  T v[V];
};

template <typename I>
__device__ __forceinline__ int64_t id_at(const void* ids, int64_t i) { return (int64_t)((const I*)ids)[i]; }
__device__ __forceinline__ int64_t id_of(const void* ids, bool wide, int64_t i) {
  return wide ? id_at<int64_t>(ids, i) : id_at<int32_t>(ids, i);
}

// ------------------------------------------------------------------------------------------
// Forward
// ------------------------------------------------------------------------------------------

struct LookUp {
  const void *table, *ids;
  void* out;
  int64_t table_stride, out_stride, rows, tokens, pieces;
  float scale;
  bool wide;
  uint32_t* status;
};

// A thread's pieces lie a block apart, so that a warp's loads and stores are of whole lines.  I: the type that holds the
// number of all pieces (32-bit divisions are several times cheaper).
template <typename T, int V, int N, typename I>
__global__ void __launch_bounds__(256) k_embed(const LookUp a) {
  const I total = (I)(a.tokens * a.pieces), first = (I)blockIdx.x * (256 * N) + threadIdx.x;
  Piece<T, V> p[N];
  I token[N], piece[N];
  bool live[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const I at = first + (I)(256 * j);
    live[j] = at < total && at >= first;
    token[j] = live[j] ? at / (I)a.pieces : 0;
    piece[j] = live[j] ? at - token[j] * (I)a.pieces : 0;
#pragma unroll
    for (int k = 0; k < V; ++k) p[j].v[k] = from_f32<T>(0.f);
    if (!live[j]) continue;
    const int64_t id = id_of(a.ids, a.wide, (int64_t)token[j]);
    if (id >= 0 && id < a.rows) p[j] = *(const Piece<T, V>*)((const T*)a.table + id * a.table_stride + (int64_t)piece[j] * V);
    else if (id != MF_NO_TOKEN && a.status) atomicOr(a.status, kStatusBadInput);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (!live[j]) continue;
#pragma unroll
    for (int k = 0; k < V; ++k) p[j].v[k] = from_f32<T>(to_f32(p[j].v[k]) * a.scale);
    *(Piece<T, V>*)((T*)a.out + (int64_t)token[j] * a.out_stride + (int64_t)piece[j] * V) = p[j];
  }
}

// ------------------------------------------------------------------------------------------
// The sort
// ------------------------------------------------------------------------------------------

constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kSortTile = 2048, kDigitBits = 10, kDigits = 1 << kDigitBits;
constexpr int kSortSteps = kSortTile / kSortThreads;  // keys of a lane
// Up to this many tiles a block adds the counts of the tiles before its own up by itself (a load of 8 bytes a tile and
// thread, 16 in flight); more are scanned by a launch of their own.
constexpr int kSortSelf = 64;

struct Sort {
  const void* ids;
  bool wide;
  int64_t tokens, rows;
  uint32_t *keys, *places;              // read (after the first pass), by the pass's order
  uint32_t *keys_out, *places_out;
  uint32_t* counts;                     // [tile][digit]
  uint32_t* totals;                     // [digit] (of scanned counts)
  uint32_t* used;                       // bit a row: some token names it
  int64_t used_words;
  uint32_t* status;
  uint32_t* crossing;                   // the number of Sums::list's units
  int shift, digits, tiles;
  bool first;
};

// A token's key: its row; those of no row (the padding of a batch, invalid ids) come last, as row `rows`.
__device__ __forceinline__ uint32_t key_at(const Sort& a, int64_t i, bool tell) {
  if (!a.first) return a.keys[i];
  const int64_t id = id_of(a.ids, a.wide, i);
  if (id >= 0 && id < a.rows) return (uint32_t)id;
  if (tell && id != MF_NO_TOKEN && a.status) atomicOr(a.status, kStatusBadInput);
  return (uint32_t)a.rows;
}

__global__ void __launch_bounds__(kSortThreads) k_embed_count(const Sort a) {
  __shared__ uint32_t s_count[kDigits];
  for (int d = threadIdx.x; d < a.digits; d += kSortThreads) s_count[d] = 0;
  if (a.first && blockIdx.x == 0 && threadIdx.x == 0) *a.crossing = 0;
  if (a.first)
    for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < a.used_words; i += (int64_t)gridDim.x * kSortThreads) a.used[i] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
  for (int j = 0; j < kSortSteps; ++j) {
    const int64_t i = lo + j * kSortThreads + threadIdx.x;
    // (one addition for a warp's equal digits: often used rows would queue)
    const uint32_t d = i < a.tokens ? (key_at(a, i, false) >> a.shift) & (a.digits - 1) : 0xFFFFFFFFu;
    const uint32_t same = __match_any_sync(0xffffffffu, d);
    if (i < a.tokens && (same & ((1u << (threadIdx.x & 31)) - 1)) == 0) atomicAdd(&s_count[d], (uint32_t)__popc(same));
  }
  __syncthreads();
  for (int d = threadIdx.x; d < a.digits; d += kSortThreads) a.counts[(int64_t)blockIdx.x * a.digits + d] = s_count[d];
}

// Counts -> how many keys of the same digit the tiles before hold, and each digit's total: 32 digits a block, 32 shares of
// the tiles each.
__global__ void __launch_bounds__(1024) k_embed_scan(uint32_t* counts, uint32_t* totals, int digits, int tiles) {
  __shared__ uint32_t s_sum[32][33];
  const int d = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5, per = (tiles + 31) / 32;
  const int lo = min(tiles, part * per), hi = min(tiles, lo + per);
  uint32_t sum = 0;
  if (d < digits)
    for (int t = lo; t < hi; ++t) sum += counts[(int64_t)t * digits + d];
  s_sum[part][threadIdx.x & 31] = sum;
  __syncthreads();
  uint32_t before = 0;
  for (int p = 0; p < part; ++p) before += s_sum[p][threadIdx.x & 31];
  if (d >= digits) return;
  for (int t = lo; t < hi; ++t) {
    uint32_t* const c = counts + (int64_t)t * digits + d;
    const uint32_t n = *c;
    *c = before;
    before += n;
  }
  if (part == 31) totals[d] = before;
}

// Exclusive sum over the block's threads.
__device__ __forceinline__ uint32_t before_me(uint32_t v, uint32_t* s_warp) {
  uint32_t sum = v;
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, sum, w);
    if ((threadIdx.x & 31) >= w) sum += o;
  }
  if ((threadIdx.x & 31) == 31) s_warp[threadIdx.x >> 5] = sum;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) base += s_warp[w];
  __syncthreads();
  return base + sum - v;
}

// Keys and places to where the pass's order has them.  Keys of one digit keep their order: tiles, warps of a tile (each
// takes consecutive keys), steps of a warp, lanes of a step.
__global__ void __launch_bounds__(kSortThreads) k_embed_scatter(const Sort a) {
  extern __shared__ __align__(4) uint16_t s_count[];  // [warp][digit]: keys of the digit in the warp, then in the warps before
  __shared__ uint32_t s_base[kDigits], s_warp[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kSortWarps * a.digits / 2; i += kSortThreads) ((uint32_t*)s_count)[i] = 0;
  if (a.first && a.tiles == 1 && threadIdx.x == 0) *a.crossing = 0;
  if (a.first && a.tiles == 1)  // (else k_embed_count has done it)
    for (int64_t i = threadIdx.x; i < a.used_words; i += kSortThreads) a.used[i] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * kSortTile + warp * (kSortTile / kSortWarps) + lane;
  uint16_t* const mine = s_count + warp * a.digits;
  uint32_t key[kSortSteps], place[kSortSteps], rank[kSortSteps];
#pragma unroll
  for (int j = 0; j < kSortSteps; ++j) {
    const int64_t i = lo + 32 * j;
    key[j] = i < a.tokens ? key_at(a, i, true) : 0xFFFFFFFFu;
    place[j] = i < a.tokens ? (a.first ? (uint32_t)i : a.places[i]) : 0u;
  }
#pragma unroll
  for (int j = 0; j < kSortSteps; ++j) {
    const bool live = lo + 32 * j < a.tokens;
    const uint32_t d = live ? (key[j] >> a.shift) & (a.digits - 1) : 0xFFFFFFFFu;
    const uint32_t same = __match_any_sync(0xffffffffu, d), before = __popc(same & ((1u << lane) - 1));
    rank[j] = live ? mine[d] + before : 0;
    __syncwarp();
    if (live && before == 0) mine[d] = (uint16_t)(mine[d] + __popc(same));
    __syncwarp();
  }
  __syncthreads();
  // thread t takes the digits 2 t and 2 t + 1
  uint32_t total[2] = {0, 0}, earlier[2] = {0, 0};
  const int d0 = 2 * threadIdx.x;
  if (d0 < a.digits) {
    uint32_t* const pairs = (uint32_t*)(s_count + d0);  // (two counts of 16 bits, of at most 2048 together)
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t n = pairs[w * a.digits / 2];
      pairs[w * a.digits / 2] = sum;
      sum += n;
    }
    if (a.tiles == 1) {
      total[0] = sum & 0xFFFFu;
      total[1] = sum >> 16;
    } else if (a.tiles <= kSortSelf) {
#pragma unroll 16
      for (int t = 0; t < a.tiles; ++t) {
        const uint2 n = *(const uint2*)(a.counts + (int64_t)t * a.digits + d0);
        if (t < (int)blockIdx.x) {
          earlier[0] += n.x;
          earlier[1] += n.y;
        }
        total[0] += n.x;
        total[1] += n.y;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        earlier[k] = a.counts[(int64_t)blockIdx.x * a.digits + d0 + k];
        total[k] = a.totals[d0 + k];
      }
    }
  }
  const uint32_t base = before_me(total[0] + total[1], s_warp);
  if (2 * threadIdx.x < (uint32_t)a.digits) {
    s_base[2 * threadIdx.x] = base + earlier[0];
    s_base[2 * threadIdx.x + 1] = base + total[0] + earlier[1];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortSteps; ++j) {
    if (lo + 32 * j >= a.tokens) continue;
    const uint32_t d = (key[j] >> a.shift) & (a.digits - 1), to = s_base[d] + mine[d] + rank[j];
    a.keys_out[to] = key[j];
    a.places_out[to] = place[j];
  }
}

// The bits of the rows that tokens name, from the sorted keys: once a row.  (Set by the sort itself, token by token, the
// often used rows of a vocabulary in order of use, which lie in few words, took 10 to 28 us.)
__global__ void __launch_bounds__(256) k_embed_mark(const uint32_t* keys, int64_t tokens, int64_t rows, uint32_t* used) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= tokens) return;
  const uint32_t key = keys[i];
  if (key < (uint32_t)rows && (i == 0 || keys[i - 1] != key)) atomicOr(used + (key >> 5), 1u << (key & 31));
}

// ------------------------------------------------------------------------------------------
// The sums
// ------------------------------------------------------------------------------------------

struct Sums {
  const uint32_t *keys, *places;
  const void* dout;
  void* out;
  float* partial;     // [unit][2][ld]: the run that a unit starts in, and the run that it ends in and has begun
  const uint32_t* used;
  int64_t dout_stride, out_stride, tokens, rows, dim, pieces, ld, units, sum_blocks;
  uint32_t* list;     // the units that begin a run which passes their end, behind their number; in no order
  int unit;           // tokens
  float scale;
};

template <typename T, int V>
__device__ __forceinline__ void write_row(const Sums& a, uint32_t row, int64_t piece, const float (&sum)[V]) {
  Piece<T, V> p;
#pragma unroll
  for (int k = 0; k < V; ++k) p.v[k] = from_f32<T>(sum[k] * a.scale);
  *(Piece<T, V>*)((T*)a.out + (int64_t)row * a.out_stride + piece * V) = p;
}

template <typename T, int V>
__global__ void __launch_bounds__(256) k_embed_sums(const Sums a) {
  if ((int64_t)blockIdx.x >= a.sum_blocks) {  // rows that no token names
    const float zero[V] = {};
    const int64_t words = (a.rows + 31) / 32;
    for (int64_t w = (int64_t)blockIdx.x - a.sum_blocks; w < words; w += (int64_t)gridDim.x - a.sum_blocks) {
      const uint32_t used = a.used[w], rows = (uint32_t)min((int64_t)32, a.rows - 32 * w);
      if (used == 0xFFFFFFFFu) continue;
      for (int64_t i = threadIdx.x; i < rows * a.pieces; i += 256) {
        const uint32_t r = (uint32_t)(a.pieces < 0x4000000 ? (uint32_t)i / (uint32_t)a.pieces : i / a.pieces);
        if (!(used >> r & 1)) write_row<T, V>(a, (uint32_t)(32 * w) + r, i - r * a.pieces, zero);
      }
    }
    return;
  }
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, unit = at / a.pieces, piece = at - unit * a.pieces;
  if (unit >= a.units) return;
  const int64_t lo = unit * a.unit, hi = min(a.tokens, lo + a.unit);
  uint32_t row = a.keys[lo];
  if (row >= (uint32_t)a.rows) return;
  bool head = lo > 0 && a.keys[lo - 1] == row;  // the run began in a unit before
  float sum[V] = {};
  float* const partial = a.partial + unit * 2 * a.ld + piece * V;
  constexpr int kAhead = 4;  // rows in flight a thread (8: twice the registers, 179 us a step of the vocabulary instead of 164)
  bool over = false;  // only tokens of no row are left
  uint32_t key[kAhead], place[kAhead];
  auto look = [&](int64_t i) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      key[j] = i + j < hi ? a.keys[i + j] : (uint32_t)a.rows;
      place[j] = i + j < hi ? a.places[i + j] : 0u;
    }
  };
  look(lo);
  for (int64_t i = lo; i < hi && !over; i += kAhead) {
    Piece<T, V> p[kAhead];
    uint32_t now[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      now[j] = key[j];
      if (key[j] < (uint32_t)a.rows) p[j] = *(const Piece<T, V>*)((const T*)a.dout + (int64_t)place[j] * a.dout_stride + piece * V);
    }
    if (i + kAhead < hi) look(i + kAhead);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i + j >= hi || over) continue;
      if (now[j] != row) {
        if (head)
#pragma unroll
          for (int k = 0; k < V; ++k) partial[k] = sum[k];
        else write_row<T, V>(a, row, piece, sum);
        head = false;
        row = now[j];
        over = row >= (uint32_t)a.rows;
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] = 0.f;
        if (over) continue;
      }
#pragma unroll
      for (int k = 0; k < V; ++k) sum[k] += to_f32(p[j].v[k]);
    }
  }
  if (over) return;
  const bool goes_on = hi < a.tokens && a.keys[hi] == row;
  if (goes_on && !head && piece == 0) a.list[1 + atomicAdd(a.list, 1u)] = (uint32_t)unit;
  if (head || goes_on) {
    float* const to = head ? partial : partial + a.ld;
#pragma unroll
    for (int k = 0; k < V; ++k) to[k] = sum[k];
  } else {
    write_row<T, V>(a, row, piece, sum);
  }
}

// Rows whose run passes a unit's border: the partial sums from the unit that begins it on.  A run over few units is added
// up in order, 128 columns a warp and 1024 a block; a longer one in eight shares of consecutive units, a warp each, and the
// shares in order, 128 columns a block.  (The longest of 61,000 tokens over 100,003 rows spans 170 units, most two or three.)
constexpr int kShortRun = 16;

template <typename T>
__device__ __forceinline__ void write_columns(const Sums& a, uint32_t row, int64_t c, const float4& sum) {
  T* const out = (T*)a.out + (int64_t)row * a.out_stride + c;
  const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < a.dim) out[k] = from_f32<T>(v[k] * a.scale);
}
__device__ __forceinline__ void add4(float4& sum, const float4& v) {
  sum.x += v.x;
  sum.y += v.y;
  sum.z += v.z;
  sum.w += v.w;
}

template <typename T>
__global__ void __launch_bounds__(256) k_embed_join(const Sums a) {
  __shared__ float4 s_sum[8][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t columns = (uint32_t)((a.dim + 127) / 128);
  const uint64_t jobs = (uint64_t)a.list[0] * columns;
  for (uint64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int64_t unit = a.list[1 + job / columns];
    const uint32_t column = (uint32_t)(job % columns), row = a.keys[(unit + 1) * a.unit];
    const int64_t at = unit + 1 + lane;
    const uint32_t near = __ballot_sync(0xffffffffu, at < a.units && a.keys[at * a.unit] == row);
    const float* const first = a.partial + (unit * 2 + 1) * a.ld;
    if (__popc(near) < kShortRun) {
      if (column % 8) continue;
      const int64_t c = ((int64_t)column + warp) * 128 + lane * 4;
      if (c >= a.dim) continue;
      float4 sum = *(const float4*)(first + c);
#pragma unroll 4
      for (int i = 1; i <= __popc(near); ++i) add4(sum, *(const float4*)(a.partial + (unit + i) * 2 * a.ld + c));
      write_columns<T>(a, row, c, sum);
      continue;
    }
    // the last unit that begins with the row: 32 candidates at a time, between one that does and one that does not
    int64_t last = unit + 1, not_it = a.units;
    while (not_it - last > 1) {
      const int64_t step = (not_it - last + 31) / 32, next = last + (lane + 1) * step;
      const uint32_t yes = __ballot_sync(0xffffffffu, next < not_it && a.keys[next * a.unit] == row);
      const int64_t most = __popc(yes);  // (sorted: those that do come first)
      not_it = min(not_it, last + (most + 1) * step);
      last += most * step;
    }
    const int64_t count = last - unit + 1, per = (count + 7) / 8, c = (int64_t)column * 128 + lane * 4, end = min(count, (warp + 1) * per);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < a.dim)
#pragma unroll 8
      for (int64_t i = warp * per; i < end; ++i) add4(sum, *(const float4*)(i ? a.partial + (unit + i) * 2 * a.ld + c : first + c));
    s_sum[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < a.dim) {
#pragma unroll
      for (int k = 1; k < 8; ++k) add4(sum, s_sum[k][lane]);
      write_columns<T>(a, row, c, sum);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------
// Few rows and tokens: no sort
// ------------------------------------------------------------------------------------------

// A block takes a row of the table and finds its tokens by itself: a list of their places, in order, in shared memory.  Then
// groups of threads take the listed rows in turn, and the groups' sums are added in pairs.  One launch
// instead of four; every block reads all ids, so it is for tables of options, not for vocabularies.
constexpr int kFewTokens = 16384, kFewThreads = 512;

template <typename T, bool VECTORS>
__global__ void __launch_bounds__(kFewThreads) k_embed_few(const void* ids, bool wide, int tokens, int64_t rows, const T* dout,
                                                           int64_t dout_stride, T* out, int64_t out_stride, int dim, float scale,
                                                           uint32_t* status) {
  constexpr int V = 4;  // columns of a thread, whatever the alignment: the order of additions does not depend on it
  __shared__ uint16_t s_list[kFewTokens];
  __shared__ float s_sum[kFewThreads][V];
  __shared__ int s_count[kFewThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = blockIdx.x;
  // a warp's tokens: `steps` times 32 in a row
  const int steps = (tokens + kFewThreads - 1) / kFewThreads, lo = warp * steps * 32;
  uint32_t mine = 0;  // lane s: which tokens of step s are the row's
  int count = 0;
  for (int s0 = 0; s0 < steps; s0 += 8) {
    int64_t id[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = lo + (s0 + k) * 32 + lane;
      id[k] = s0 + k < steps && i < tokens ? id_of(ids, wide, i) : MF_NO_TOKEN;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t m = __ballot_sync(0xffffffffu, id[k] == row);
      if (lane == s0 + k) mine = m;
      count += __popc(m);
      if (row == 0 && blockIdx.y == 0 && status && id[k] != MF_NO_TOKEN && (id[k] < 0 || id[k] >= rows)) atomicOr(status, kStatusBadInput);
    }
  }
  if (lane == 0) s_count[warp] = count;
  __syncthreads();
  int at = 0, all = 0;
  for (int w = 0; w < kFewThreads / 32; ++w) {
    if (w < warp) at += s_count[w];
    all += s_count[w];
  }
  for (int s = 0; s < steps; ++s) {
    const uint32_t m = __shfl_sync(0xffffffffu, mine, s);
    if (m >> lane & 1) s_list[at + __popc(m & ((1u << lane) - 1))] = (uint16_t)(lo + s * 32 + lane);
    at += __popc(m);
  }
  __syncthreads();
  // a group: the threads of up to 128 columns (a power of two of them)
  int width = 1;
  while (width * V < dim && width < 32) width *= 2;
  const int groups = kFewThreads / width, group = threadIdx.x / width;
  const int c = (blockIdx.y * 32 + threadIdx.x % width) * V;
  float sum[V] = {};
  if (c < dim) {
#pragma unroll 4
    for (int i = group; i < all; i += groups) {
      const T* const from = dout + (int64_t)s_list[i] * dout_stride + c;
      Piece<T, V> p;
      if constexpr (VECTORS) p = *(const Piece<T, V>*)from;
      else
#pragma unroll
        for (int k = 0; k < V; ++k) p.v[k] = c + k < dim ? from[k] : from_f32<T>(0.f);
#pragma unroll
      for (int k = 0; k < V; ++k) sum[k] += to_f32(p.v[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) s_sum[threadIdx.x][k] = sum[k];
  for (int half = groups / 2; half > 0; half /= 2) {
    __syncthreads();
    if (group < half)
#pragma unroll
      for (int k = 0; k < V; ++k) s_sum[threadIdx.x][k] += s_sum[threadIdx.x + half * width][k];
  }
  if (group == 0)
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + k < dim) out[row * out_stride + c + k] = from_f32<T>(s_sum[threadIdx.x][k] * scale);
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------

// Values of a piece: the most, up to 16 bytes, that rows of `dim` values at these addresses and strides divide into.
int piece_of(int size, int64_t dim, const void* a, int64_t sa, const void* b, int64_t sb) {
  int v = 16 / size;
  while (v > 1 && (dim % v || sa % v || sb % v || ((uintptr_t)a | (uintptr_t)b) % (size_t)(v * size))) v /= 2;
  return v;
}

// Whether a call goes without a sort: where all blocks together read few ids, and the values fill no GPU.  (48 rows of 8
// fp32 values, 10240 tokens: 11 us on the device and 23 a call with the lookup; by the sort 43 and 41.)
bool few_of(const mf_embedding_grad_args& p) {
  return p.tokens <= kFewTokens && p.rows <= 65536 && p.dim <= 65536 && p.tokens * p.dim <= (1 << 21) &&
         p.rows * ((p.dim + 127) / 128) * (p.tokens + 256) <= (1 << 22);
}

template <typename T>
mf_status few(const mf_embedding_grad_args& p, cudaStream_t s) {
  const bool vectors = piece_of(sizeof(T), p.dim, p.d_dout, p.dout_stride, p.d_dtable, p.dtable_stride) >= 4;
  const dim3 grid((unsigned)p.rows, (unsigned)((p.dim + 127) / 128));
  auto kernel = vectors ? k_embed_few<T, true> : k_embed_few<T, false>;
  kernel<<<grid, kFewThreads, 0, s>>>(p.d_ids, p.id_bits == 64, (int)p.tokens, p.rows, (const T*)p.d_dout, p.dout_stride, (T*)p.d_dtable,
                                      p.dtable_stride, (int)p.dim, p.scale, p.d_status);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

template <typename T, int V>
mf_status look_up(const mf_embedding_args& p, const LookUp& a, cudaStream_t s) {
  const int64_t total = a.tokens * a.pieces;
  if (total < (int64_t(1) << 31)) {
    // few pieces: one a thread, on more SMs
    if (total <= 152 * 2048) k_embed<T, V, 1, uint32_t><<<(unsigned)((total + 255) / 256), 256, 0, s>>>(a);
    else k_embed<T, V, 4, uint32_t><<<(unsigned)((total + 1023) / 1024), 256, 0, s>>>(a);
  } else {
    const int64_t blocks = (total + 1023) / 1024;
    if (blocks > 0x7FFFFFFF) {
      set_error("mf_embedding: tokens * dim is too large");
      return MF_EINVAL;
    }
    k_embed<T, V, 4, uint64_t><<<(unsigned)blocks, 256, 0, s>>>(a);
  }
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

struct GradPlan {
  int bits, passes, digit_bits, tiles, unit;
  int64_t units, ld, used_words;
  int64_t keys[2], places[2], counts, totals, used, list, partial, bytes;  // offsets of the scratch memory
};

GradPlan grad_plan(const mf_embedding_grad_args& p) {
  GradPlan g{};
  g.bits = 1;
  while (g.bits < 32 && ((uint64_t)p.rows >> g.bits)) ++g.bits;  // keys are 0..rows
  g.passes = (g.bits + kDigitBits - 1) / kDigitBits;
  g.digit_bits = (g.bits + g.passes - 1) / g.passes;
  g.tiles = (int)((p.tokens + kSortTile - 1) / kSortTile);
  // A unit: enough threads in all to fill the GPU, and at most 8192 units for the sums of a row that all tokens name.
  // (By 8 values as most calls go; how rows are aligned changes no order of additions.)
  const int64_t pieces = (p.dim + 7) / 8;
  const double fill = (double)p.tokens * (double)pieces / 300000.0;
  g.unit = (int)std::max(fill >= 32.0 ? (int64_t)32 : std::max((int64_t)fill, (int64_t)8), (p.tokens + 8191) / 8192);
  g.units = (p.tokens + g.unit - 1) / g.unit;
  g.ld = (p.dim + 7) / 8 * 8;
  g.used_words = (p.rows + 31) / 32;
  int64_t at = 0;
  auto take = [&at](int64_t bytes) {
    const int64_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  for (int k = 0; k < 2; ++k) {
    g.keys[k] = take(4 * p.tokens);
    g.places[k] = take(4 * p.tokens);
  }
  g.counts = take((int64_t)4 * g.tiles << g.digit_bits);
  g.totals = take(4 << g.digit_bits);
  g.used = take(4 * g.used_words);
  g.list = take(4 * (g.units + 1));
  g.partial = take(8 * g.units * g.ld);
  g.bytes = at;
  return g;
}

template <typename T, int V>
mf_status sums(const Sums& a, cudaStream_t s) {
  Sums b = a;
  b.pieces = a.dim / V;
  b.sum_blocks = (b.units * b.pieces + 255) / 256;
  // the rows to be zeroed: 32 a block at a time
  const int64_t zero_blocks = std::min((b.rows + 31) / 32, (int64_t)(152 * 16));
  if (b.sum_blocks + zero_blocks > 0x7FFFFFFF) {
    set_error("mf_embedding_backward: tokens * dim is too large");
    return MF_EINVAL;
  }
  k_embed_sums<T, V><<<(unsigned)(b.sum_blocks + zero_blocks), 256, 0, s>>>(b);
  MF_CUDA(cudaGetLastError());
  if (b.units > 1) {
    k_embed_join<T><<<(unsigned)std::min(b.units * ((b.dim + 127) / 128), (int64_t)(152 * 8)), 256, 0, s>>>(b);
    MF_CUDA(cudaGetLastError());
  }
  return MF_OK;
}

}  // namespace

mf_status embed_forward(const mf_embedding_args& p, cudaStream_t s) {
  LookUp a{p.d_table, p.d_ids, p.d_out, p.table_stride, p.out_stride, p.rows, p.tokens, 0, p.scale, p.id_bits == 64, p.d_status};
  const int size = p.type == MF_TYPE_F32 ? 4 : 2, v = piece_of(size, p.dim, p.d_table, p.table_stride, p.d_out, p.out_stride);
  a.pieces = p.dim / v;
  if (size == 4) return v == 4 ? look_up<float, 4>(p, a, s) : v == 2 ? look_up<float, 2>(p, a, s) : look_up<float, 1>(p, a, s);
  if (p.type == MF_TYPE_BF16)
    return v == 8 ? look_up<__nv_bfloat16, 8>(p, a, s) : v == 4 ? look_up<__nv_bfloat16, 4>(p, a, s) :
           v == 2 ? look_up<__nv_bfloat16, 2>(p, a, s) : look_up<__nv_bfloat16, 1>(p, a, s);
  return v == 8 ? look_up<__half, 8>(p, a, s) : v == 4 ? look_up<__half, 4>(p, a, s) :
         v == 2 ? look_up<__half, 2>(p, a, s) : look_up<__half, 1>(p, a, s);
}

uint64_t embed_work(const mf_embedding_grad_args& p) {
  if (few_of(p)) return 0;
  return p.tokens ? (uint64_t)grad_plan(p).bytes : (uint64_t)(4 * ((p.rows + 31) / 32));
}

mf_status embed_backward(const mf_embedding_grad_args& p, void* work, cudaStream_t s) {
  if (few_of(p)) return p.type == MF_TYPE_F32 ? few<float>(p, s) : p.type == MF_TYPE_BF16 ? few<__nv_bfloat16>(p, s) : few<__half>(p, s);
  char* const w = (char*)work;
  Sums b{};
  b.dout = p.d_dout;
  b.out = p.d_dtable;
  b.dout_stride = p.dout_stride;
  b.out_stride = p.dtable_stride;
  b.tokens = p.tokens;
  b.rows = p.rows;
  b.dim = p.dim;
  b.scale = p.scale;
  if (p.tokens) {
    const GradPlan g = grad_plan(p);
    Sort a{};
    a.ids = p.d_ids;
    a.wide = p.id_bits == 64;
    a.tokens = p.tokens;
    a.rows = p.rows;
    a.status = p.d_status;
    a.counts = (uint32_t*)(w + g.counts);
    a.totals = (uint32_t*)(w + g.totals);
    a.used = (uint32_t*)(w + g.used);
    a.used_words = g.used_words;
    a.crossing = (uint32_t*)(w + g.list);
    a.digits = 1 << g.digit_bits;
    a.tiles = g.tiles;
    for (int k = 0; k < g.passes; ++k) {
      a.first = k == 0;
      a.shift = k * g.digit_bits;
      a.keys = (uint32_t*)(w + g.keys[k & 1]);
      a.places = (uint32_t*)(w + g.places[k & 1]);
      a.keys_out = (uint32_t*)(w + g.keys[~k & 1]);
      a.places_out = (uint32_t*)(w + g.places[~k & 1]);
      if (g.tiles > 1) {
        k_embed_count<<<g.tiles, kSortThreads, 0, s>>>(a);
        MF_CUDA(cudaGetLastError());
      }
      if (g.tiles > kSortSelf) {
        k_embed_scan<<<(a.digits + 31) / 32, 1024, 0, s>>>(a.counts, a.totals, a.digits, g.tiles);
        MF_CUDA(cudaGetLastError());
      }
      k_embed_scatter<<<g.tiles, kSortThreads, 2 * kSortWarps * a.digits, s>>>(a);
      MF_CUDA(cudaGetLastError());
    }
    k_embed_mark<<<(unsigned)((p.tokens + 255) / 256), 256, 0, s>>>(a.keys_out, p.tokens, p.rows, a.used);
    MF_CUDA(cudaGetLastError());
    b.keys = a.keys_out;
    b.places = a.places_out;
    b.used = a.used;
    b.list = a.crossing;
    b.partial = (float*)(w + g.partial);
    b.unit = g.unit;
    b.units = g.units;
    b.ld = g.ld;
  } else {
    MF_CUDA(cudaMemsetAsync(w, 0, 4 * ((p.rows + 31) / 32), s));
    b.used = (const uint32_t*)w;
  }
  const int size = p.type == MF_TYPE_F32 ? 4 : 2;
  const int v = piece_of(size, p.dim, p.d_dout, p.dout_stride, p.d_dtable, p.dtable_stride);
  if (size == 4) return v == 4 ? sums<float, 4>(b, s) : v == 2 ? sums<float, 2>(b, s) : sums<float, 1>(b, s);
  if (p.type == MF_TYPE_BF16)
    return v == 8 ? sums<__nv_bfloat16, 8>(b, s) : v == 4 ? sums<__nv_bfloat16, 4>(b, s) :
           v == 2 ? sums<__nv_bfloat16, 2>(b, s) : sums<__nv_bfloat16, 1>(b, s);
  return v == 8 ? sums<__half, 8>(b, s) : v == 4 ? sums<__half, 4>(b, s) : v == 2 ? sums<__half, 2>(b, s) : sums<__half, 1>(b, s);
}

}  // namespace mf
