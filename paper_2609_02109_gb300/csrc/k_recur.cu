// Gated linear recurrence over sequences and its gradient (the operators' section of include/mf.h).
//
// h_t = f_t h_{t-1} + g_t x_t is a chain of maps s -> A s + B, and maps compose: (A2, B2) after (A1, B1) is
// (A2 A1, A2 B1 + B2).  The gradient is such a chain too, from the last step to the first, on the value b
// that a step passes back: b <- f_t (dh_t + b).  The kernel below, in either direction, is one pass over the data:
//
//   a thread holds one 32-bit word (one fp32 channel, or two 16-bit ones) of 16 steps in registers;
//   the lanes of a row of `lc` words (32 where there are as many) lie side by side, so a warp reads and writes whole
//   sectors;
//   a block of up to 256 threads holds a tile of (256 / lc) segments of 16 steps, scans the segments'
//   maps (shuffles within a warp, shared memory between warps), and then walks its 16 steps with the
//   state that reaches them.
//
// A chain (a batch row's group of lc words) is walked tile after tile by one block where there are chains
// enough to fill the GPU.  Else `ways` blocks share it: in each round they take neighbouring tiles, tell each other
// their tiles' maps and fold those of the round in order, so equal calls give equal bits.  Up to 4 blocks are a
// cluster and write their maps into each other's shared memory; where chains are too few for that to occupy the
// GPU, more blocks (all resident: a cooperative launch) publish them in global memory, two or three L2 round trips
// (2-4 us) a round.  The next tile's words are copied to shared memory before the wait: rows of 32 words by one
// tensor copy (TMA) a tensor, narrower ones by cp.async; short sequences and rows that are not whole words are
// read straight from memory.
//
// Bound: memory, 3 words read and written per word of x forward, 5 backward (x and z again, since the rest
// of a network ran between); the backward call starts each segment from the state that the forward call
// saved for it (4 bytes for 16 steps of a channel), so it needs h neither in memory nor rounded.  Issue slots are
// nearly as scarce (24 instructions an element forward, 16-bit, 46 backward), hence packed fp32 pairs and loops without conditions.
// Measured (cold caches, launch included), of the measured copy rate: bf16 32 x 2048 x 2048 forward 138 us (0.87) and 242
// backward (0.83), 8 x 8192 x 2048 148 us (0.81) and 267 (0.75), f16 8 x 4096 x 2048 80 us (0.75) and 140 (0.72); f32 8 x 4096 x
// 2048 160 us (0.75) and 201 (1.0); where chains are shared, f16 1 x 65536 x 4096 359 us (0.67) and f32 1 x 200003 x 512
// 267 us (0.69) and 384 (0.80): a round's exchange is not hidden.  16-bit rows of an odd width, straight from memory: bf16
// 64 x 100 x 2047 134 us and 189, where 2048 take 35 and 48.
#include <type_traits>

#include "mf_ops.cuh"
#include "tma.cuh"

namespace mf {
namespace {

constexpr int kSeg = kRecurSave;   // steps of a thread
constexpr int kMostThreads = 256;
constexpr int kMostCluster = 4;
constexpr float kTiny = 0x1p-149f;  // least factor of a map that cuts nothing (see Map)
constexpr uint32_t kTries = 4096;  // of a bounded wait: tests of a barrier (a millisecond each at most), or 1024 polls of L2

struct Seq {
  char* p;
  int64_t sb, st;  // bytes
};

struct Args {
  int64_t batch, time, dim;
  Seq x, z, y, dx, dz;   // y: h (forward) or dh (backward)
  const uint8_t* marks;
  int64_t mb, mt;
  bool marks16;          // a segment's 16 marks are one aligned 16-byte word
  const float* first;    // h0, or dlast: [batch][dim] or NULL
  float* end;            // last, or dh0
  float* saved;
  ulonglong2* maps;      // [chain][2][ways][channels of a row]: published maps (see publish)
  uint32_t* status;
  uint32_t tries;        // of a bounded wait
  uint32_t unsent;       // bytes that waits expect and nothing sends (mf_debug_operators_wait_test; else 0)
  int64_t tiles;
  int groups, lc, ways;
  bool cluster;          // ways > 1: the chain's blocks are a cluster
  bool whole;            // rows start and end on words
};

// s -> a s + b.  a is 0 only where a first sample cuts the chain, and then nothing of s passes, not even a
// NaN or an infinity.  Factors that underflow, or are 0, stay at kTiny, so that they do not cut: an infinity passes, and of
// a finite state s at most 2^-149 |s| <= 4.8e-7.
struct Map {
  float a, b;
};
__device__ __forceinline__ float through(Map m, float s) { return m.a == 0.f ? m.b : fmaf(m.a, s, m.b); }
__device__ __forceinline__ Map after(Map m2, Map m1) {  // first m1, then m2
  const float a = m2.a * m1.a;
  return {m2.a == 0.f || m1.a == 0.f ? 0.f : fmaxf(a, kTiny), through(m2, m1.b)};
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{.reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 z, x, y;\n mov.b64 {%0, %1}, z;}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{.reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 z, x, y;\n mov.b64 {%0, %1}, z;}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// The gates f = 1 / (1 + e^-z) and g = 1 - f of two values: with e = e^-|z|, the larger of f and g is 1 / (1 + e)
// and the smaller e / (1 + e), so neither cancels or overflows.  The hardware's 2^x and 1 / x (errors of about
// 2^-22) and one rounding of z log2 e: relative errors of at most (|z| + 6) 2^-24, which a state's memory averages;
// the library's expf, exact to 2^-23, takes three times the instructions, and issue slots are as scarce here as bandwidth.
__device__ __forceinline__ void gate2(float2 z, float2& small, float2& large) {
  const float2 t = mul2(z, make_float2(1.4426950408889634f, 1.4426950408889634f));
  float2 e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(-fabsf(t.x)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(-fabsf(t.y)));
  const float2 d = add2(e, make_float2(1.f, 1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(large.x) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(large.y) : "f"(d.y));
  small = mul2(e, large);
}

// f and g as one number: the smaller one, with the sign bit where that is f (it may be 0).  Both come back to within
// a rounding.
__device__ __forceinline__ float pack_gate(float small, float z) { return copysignf(small, z); }
__device__ __forceinline__ float gate_f(float p) { return __float_as_int(p) < 0 ? -p : 1.f - p; }
__device__ __forceinline__ float gate_g(float p) { return __float_as_int(p) < 0 ? 1.f + p : p; }

template <typename T> struct Words;
template <> struct Words<float> {
  static constexpr int V = 1;
  static constexpr uint32_t kInf = 0x7F800000u;
  static __device__ __forceinline__ void open(uint32_t w, float (&v)[1]) { v[0] = __uint_as_float(w); }
  static __device__ __forceinline__ uint32_t close(const float (&v)[1]) { return __float_as_uint(v[0]); }
};
template <> struct Words<__nv_bfloat16> {
  static constexpr int V = 2;
  static constexpr uint32_t kInf = 0x7F807F80u;
  static __device__ __forceinline__ void open(uint32_t w, float (&v)[2]) {
    v[0] = __uint_as_float(w << 16);
    v[1] = __uint_as_float(w & 0xFFFF0000u);
  }
  static __device__ __forceinline__ uint32_t close(const float (&v)[2]) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
};
template <> struct Words<__half> {
  static constexpr int V = 2;
  static constexpr uint32_t kInf = 0x7C007C00u;
  static __device__ __forceinline__ void open(uint32_t w, float (&v)[2]) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w));
    v[0] = p.x;
    v[1] = p.y;
  }
  static __device__ __forceinline__ uint32_t close(const float (&v)[2]) {
    const __half2 p = __floats2half2_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
};

__device__ __forceinline__ void copy_word(uint32_t* to, const char* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
template <int LEFT>
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }  // but the last groups
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// A word; `whole` unless it is two 16-bit channels whose address may be odd, or whose second channel may not exist.
__device__ __forceinline__ uint32_t load_word(const char* p, bool whole, bool second) {
  if (whole) return *reinterpret_cast<const uint32_t*>(p);
  const uint32_t lo = *reinterpret_cast<const uint16_t*>(p);
  return second ? lo | ((uint32_t)*reinterpret_cast<const uint16_t*>(p + 2) << 16) : lo;
}
__device__ __forceinline__ void store_word(char* p, uint32_t w, bool whole, bool second) {
  if (whole) {
    *reinterpret_cast<uint32_t*>(p) = w;
    return;
  }
  *reinterpret_cast<uint16_t*>(p) = (uint16_t)w;
  if (second) *reinterpret_cast<uint16_t*>(p + 2) = (uint16_t)(w >> 16);
}

// A published map: a and b, each in a 64-bit word with the round's tag, so that a reader needs no flag and no fence: it
// polls the words themselves, and each is written and read whole.
__device__ __forceinline__ void publish(ulonglong2* to, Map m, uint32_t tag) {
  const unsigned long long t = (unsigned long long)tag << 32;
  asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(to), "l"(t | __float_as_uint(m.a)),
               "l"(t | __float_as_uint(m.b)) : "memory");
}
__device__ __forceinline__ bool published(const ulonglong2* from, uint32_t tag, Map& m) {
  unsigned long long a, b;
  asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "l"(from) : "memory");
  m = {__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)b)};
  return (uint32_t)(a >> 32) == tag && (uint32_t)(b >> 32) == tag;
}

__device__ __forceinline__ char* row_of(char* p, int64_t stride, int i) { return p + stride * i; }

// Tiles whose words are in shared memory or on the way there.
template <typename T, bool BACK> __host__ __device__ constexpr int buffers() { return !BACK && sizeof(T) == 2 ? 2 : 1; }
// Blocks of an SM.  Forward, 16-bit: 64 registers of (f, g x) a thread; backward 64 (gate, dz / l).
template <typename T, bool BACK> constexpr int blocks_per_sm() { return sizeof(T) == 4 ? (BACK ? 2 : 3) : 2; }

// What a warp's segments hold (see `kind`): samples alone; samples and missing ones; first samples too; or not every step.
enum Kind { kPlain, kMissing, kWhole, kAny };

// How a tile's words come in.  kTensor: rows of 32 words by tensor copies (rows on 16 bytes).  kWords: every row starts
// on a word and ends with one, so that words are copied whole.  kDirect: straight from memory,
// where a block is smaller (short sequences) or rows are not whole words (16-bit loads and stores).
enum Load { kTensor, kWords, kDirect };

struct Maps3 {
  CUtensorMap x, z, y;
};

// The rest of a bounded wait, out of line: on giving up it flags the status word, and later waits return at once.
__device__ __noinline__ void wait_more(uint64_t* bar, uint32_t parity, volatile int* gave_up, uint32_t tries, uint32_t* status) {
  if (*gave_up || barrier_wait(bar, parity, tries)) return;
  *gave_up = 1;
  if (status) atomicOr(status, kStatusTimeout);
}

// The map of a tile: its warps' maps one after the other, in pairs (three dependent steps, not seven).
__device__ __forceinline__ Map tile_map(const Map (*warps)[32], int col, int nwarp) {
  Map m[kMostThreads / 32];
#pragma unroll
  for (int w = 0; w < kMostThreads / 32; ++w) m[w] = w < nwarp ? warps[w][col] : Map{1.f, 0.f};
#pragma unroll
  for (int d = 1; d < kMostThreads / 32; d *= 2)
#pragma unroll
    for (int w = 0; w + d < kMostThreads / 32; w += 2 * d) m[w] = after(m[w + d], m[w]);
  return m[0];
}

template <typename T, bool BACK, int LOAD, bool MARKS>
__global__ void __launch_bounds__(kMostThreads, blocks_per_sm<T, BACK>()) k_recur(const Args a, const __grid_constant__ Maps3 maps3) {
  constexpr bool VEC = LOAD != kDirect;
  constexpr int kTileWords = kSeg * kMostThreads, kBufs = buffers<T, BACK>();  // of one tensor in shared memory
  using W = Words<T>;
  constexpr int V = W::V;
  // the words of kBufs tiles, the rounds' in turn; kTensor: [tensor][step of the tile][32]; kWords: [tensor][step of the segment][thread]
  extern __shared__ uint32_t s_raw[];
  uint32_t* const s_words = s_raw + ((128 - (shared_u32(s_raw) & 127)) & 127) / 4;  // (tensor copies write from 128 bytes on)
  __shared__ uint64_t s_bar[2];
  __shared__ Map s_warp[2][V][kMostThreads / 32][32];   // [tile parity]: maps of the warps' segments
  // cluster: [round's parity] the round's maps; else with ways > 1 maps of parts of a round, and of what precedes the tile
  constexpr int kRowMaps = 32 * V, kClusterMaps = 2 * kMostCluster * kRowMaps, kPartMaps = kMostThreads + kRowMaps;
  __shared__ Map s_round[kClusterMaps > kPartMaps ? kClusterMaps : kPartMaps];
  __shared__ uint64_t s_told[2];
  __shared__ int s_gave_up;

  const int tid = threadIdx.x, nthr = blockDim.x, lc = LOAD == kTensor ? 32 : a.lc;
  const int col = LOAD == kTensor ? (tid & 31) : tid % lc;
  const int lseg = LOAD == kTensor ? (tid >> 5) : tid / lc, nseg = LOAD == kTensor ? (nthr >> 5) : nthr / lc;  // lseg: in the chain's order
  const int lane = tid & 31, warp = tid >> 5, nwarp = nthr >> 5;
  const int seg = BACK ? nseg - 1 - lseg : lseg;               // in time
  const int way = (int)(blockIdx.x % a.ways);
  const int64_t chain = blockIdx.x / a.ways;
  const int64_t b = chain / a.groups, c0 = ((chain % a.groups) * lc + col) * V;
  const bool live = c0 < a.dim, second = V == 1 || c0 + 1 < a.dim;
  const int64_t nsave = (a.time + kSeg - 1) / kSeg;
  if (tid == 0) {
    s_gave_up = 0;
    barrier_init(&s_bar[0], 1);
    barrier_init(&s_bar[1], 1);
    barrier_init(&s_told[0], 1);
    barrier_init(&s_told[1], 1);
    barrier_init_fence();
  }
  __syncthreads();
  if (a.cluster) cluster_sync();
  // this thread's word of step 0 of its segment in shared memory, and from step to step
  constexpr int kStep = LOAD == kTensor ? 32 : kMostThreads;
  const uint32_t* mine_w = s_words + (LOAD == kTensor ? seg * kSeg * 32 + col : tid);

  const char* px = a.x.p + b * a.x.sb + c0 * (int64_t)sizeof(T);
  const char* pz = a.z.p + b * a.z.sb + c0 * (int64_t)sizeof(T);
  char* py = a.y.p + b * a.y.sb + c0 * (int64_t)sizeof(T);
  char* pdx = BACK ? a.dx.p + b * a.dx.sb + c0 * (int64_t)sizeof(T) : nullptr;
  char* pdz = BACK ? a.dz.p + b * a.dz.sb + c0 * (int64_t)sizeof(T) : nullptr;

  // the chain's state before its tile (in the chain's order), as far as it is known
  float state[V];
#pragma unroll
  for (int v = 0; v < V; ++v) state[v] = live && (v == 0 || second) && a.first ? a.first[b * a.dim + c0 + v] : 0.f;

  // first step and number of steps of this thread's segment in a tile
  auto segment = [&](int64_t tile, int64_t& t0) -> int {
    t0 = ((BACK ? a.tiles - 1 - tile : tile) * nseg + seg) * kSeg;
    const int64_t left = a.time - t0;
    return !live || left <= 0 ? 0 : (int)(left < kSeg ? left : kSeg);
  };
  // a tile's words to shared memory, kBufs rounds ahead; dh has two places (the round's parity)
  constexpr int kBufWords = 2 * kTileWords;
  auto fetch = [&](int64_t tile, int buf, int par) {
    if constexpr (LOAD == kTensor) {  // (every thread has read its words of the tile before)
      if (tid == 0 && tile < a.tiles) {
        const int32_t e0 = (int32_t)(chain % a.groups) * 32 * V, e2 = (int32_t)b;
        const int32_t e1 = (int32_t)((BACK ? a.tiles - 1 - tile : tile) * nseg * kSeg);
        uint32_t* const to = s_words + buf * kBufWords;
        barrier_expect(&s_bar[buf], (BACK ? 3 : 2) * (uint32_t)nthr * kSeg * 4 + a.unsent);
        tma_load_3d(to, &maps3.x, e0, e1, e2, &s_bar[buf]);
        tma_load_3d(to + kTileWords, &maps3.z, e0, e1, e2, &s_bar[buf]);
        if constexpr (BACK) tma_load_3d(s_words + (2 + par) * kTileWords, &maps3.y, e0, e1, e2, &s_bar[buf]);
      }
    }
    if constexpr (LOAD == kWords) {
      int64_t t0;
      const int n = tile < a.tiles ? segment(tile, t0) : 0;
      if (n) {
        const char *qx = px + t0 * a.x.st, *qz = pz + t0 * a.z.st, *qy = BACK ? py + t0 * a.y.st : nullptr;
        uint32_t* to = s_words + buf * kBufWords + tid;
#pragma unroll
        for (int i = 0; i < kSeg; ++i) {
          if (i < n) {
            copy_word(to + i * kMostThreads, qx);
            copy_word(to + kTileWords + i * kMostThreads, qz);
            if constexpr (BACK) copy_word(s_words + tid + (2 + par) * kTileWords + i * kMostThreads, qy);
          }
          qx += a.x.st;
          qz += a.z.st;
          if constexpr (BACK) qy += a.y.st;
        }
      }
      copies_end();
    }
  };
  // its marks and saved states to registers; a round ahead
  uint32_t marks[4], saved_w[V];
  auto fetch_side = [&](int64_t tile) {
    int64_t t0;
    const int n = tile < a.tiles ? segment(tile, t0) : 0;
    if constexpr (MARKS) {
      marks[0] = marks[1] = marks[2] = marks[3] = 0x01010101u;
      if (n) {
        const uint8_t* pm = a.marks + b * a.mb + t0 * a.mt;
        if (n == kSeg && a.marks16) {
          const uint4 w = *reinterpret_cast<const uint4*>(pm);
          marks[0] = w.x; marks[1] = w.y; marks[2] = w.z; marks[3] = w.w;
        } else {
#pragma unroll
          for (int i = 0; i < kSeg; ++i) {
            const uint32_t m = i < n ? pm[i * a.mt] : 1u;
            marks[i / 4] = (marks[i / 4] & ~(0xFFu << (8 * (i & 3)))) | m << (8 * (i & 3));
          }
        }
      }
    }
    if constexpr (BACK) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        saved_w[v] = n && (v == 0 || second) ? __float_as_uint(a.saved[(b * nsave + t0 / kSeg) * a.dim + c0 + v]) : 0u;
    }
  };

  int64_t tile = way;
#pragma unroll
  for (int i = 0; i < kBufs; ++i) fetch(tile + i * a.ways, i, i);
  fetch_side(tile);
  for (uint32_t round = 0; (int64_t)round * a.ways < a.tiles; ++round, tile += a.ways) {
    int64_t t0;
    const int n = tile < a.tiles ? segment(tile, t0) : 0;
    // forward: p = f, q = g x.  backward: p = the gate, q = dz / l.  Steps that are not there: f = 1, q = 0.
    float p[kSeg][V], q[kSeg][V];
    uint32_t firsts = 0, gone = 0;  // bits of the segment's steps
    const int par = round & 1, buf = kBufs == 2 ? par : 0;
    if constexpr (LOAD == kWords) copies_done<kBufs - 1>();
    if constexpr (LOAD == kTensor) {
      const uint32_t parity = (kBufs == 2 ? round >> 1 : round) & 1;
      if (tile < a.tiles && !barrier_test(&s_bar[buf], parity)) wait_more(&s_bar[buf], parity, &s_gave_up, a.tries, a.status);
    }
    if constexpr (MARKS) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // four marks at a time: all-ones bytes, then one bit of each
        const uint32_t out4 = __vcmpeq4(marks[k], 0u), first4 = __vcmpeq4(marks[k], 0x01010101u * MF_MARK_FIRST);
        gone |= (((out4 & 0x08040201u) * 0x01010101u) >> 24) << (4 * k);
        firsts |= (((first4 & 0x08040201u) * 0x01010101u) >> 24) << (4 * k);
      }
    }
    gone |= ~0u << n;
    int kind = kPlain;
    if (!VEC || !__all_sync(0xffffffffu, n == kSeg)) kind = kAny;
    else if (MARKS && __any_sync(0xffffffffu, firsts != 0)) kind = kWhole;
    else if (MARKS && __any_sync(0xffffffffu, (gone & ((1u << kSeg) - 1)) != 0)) kind = kMissing;
    Map mine[V];
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      mine[v] = {1.f, 0.f};
      h[v] = BACK ? __uint_as_float(saved_w[v]) : 0.f;
    }
    const uint32_t* const words = mine_w + buf * kBufWords;
    // dh of a step (read where it is used: registers are short)
    [[maybe_unused]] const uint32_t* const dh_words = mine_w + (2 + par) * kTileWords;
    const auto dh_word = [&](bool there, int i) -> uint32_t {
      if (!there) return 0u;
      if constexpr (VEC) return dh_words[i * kStep];
      else return load_word(py + (t0 + i) * a.y.st, sizeof(T) == 4 || a.whole, second);
    };
    const auto walk = [&](auto kind_of) {
      constexpr int KIND = decltype(kind_of)::value;
      [[maybe_unused]] const char *qx = px, *qz = pz;
      if constexpr (!VEC) {
        if (n) {
          qx += t0 * a.x.st;
          qz += t0 * a.z.st;
        }
      }
      constexpr int J = 2 / V;  // steps of a pair
#pragma unroll
      for (int i0 = 0; i0 < kSeg; i0 += J) {
        float x[2], z[2];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int i = i0 + j;
          uint32_t wx = 0, wz = 0;
          if (KIND != kAny || i < n) {
            if constexpr (VEC) {
              wx = words[i * kStep];
              wz = words[kTileWords + i * kStep];
            } else {
              wx = load_word(qx, sizeof(T) == 4 || a.whole, second);
              wz = load_word(qz, sizeof(T) == 4 || a.whole, second);
            }
          }
          if constexpr (!VEC) {
            qx += a.x.st;
            qz += a.z.st;
          }
          if (KIND != kPlain && ((gone >> i) & 1u)) {  // z = infinity, x = 0: f = 1, 1 - f = 0, nothing added
            wx = 0u;
            wz = W::kInf;
          }
          float ox[V], oz[V];
          W::open(wx, ox);
          W::open(wz, oz);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            x[j * V + v] = ox[v];
            z[j * V + v] = oz[v];
          }
        }
        float2 small, large;
        gate2(make_float2(z[0], z[1]), small, large);
        const float2 fg = mul2(small, large);
        const float2 g = make_float2(z[0] < 0.f ? large.x : small.x, z[1] < 0.f ? large.y : small.y);
        float2 in = mul2(g, make_float2(x[0], x[1]));
        float2 f = make_float2(z[0] < 0.f ? small.x : large.x, z[1] < 0.f ? small.y : large.y);
        float2 gate = BACK ? make_float2(pack_gate(small.x, z[0]), pack_gate(small.y, z[1])) : f;
        constexpr bool kFirsts = MARKS && (KIND == kWhole || KIND == kAny);
        const bool first[2] = {kFirsts && ((firsts >> i0) & 1u), kFirsts && ((firsts >> (i0 + J - 1)) & 1u)};
        if constexpr (!BACK) {
          if (first[0]) gate.x = f.x = 0.f;
          if (first[1]) gate.y = f.y = 0.f;
          p[i0][0] = gate.x; p[i0 + J - 1][V - 1] = gate.y;
          q[i0][0] = in.x; q[i0 + J - 1][V - 1] = in.y;
        } else {
          p[i0][0] = gate.x; p[i0 + J - 1][V - 1] = gate.y;
        }
        if constexpr (V == 2) {
          if constexpr (!BACK) {
            if (first[0]) mine[0].b = mine[1].b = 0.f;
            const float2 mb = fma2(f, make_float2(mine[0].b, mine[1].b), in), ma = mul2(f, make_float2(mine[0].a, mine[1].a));
            mine[0] = {ma.x, mb.x};
            mine[1] = {ma.y, mb.y};
          } else {
            if (first[0]) h[0] = h[1] = 0.f;
            const float2 before = make_float2(h[0], h[1]);
            const float2 qq = mul2(add2(before, make_float2(-x[0], -x[1])), fg);
            q[i0][0] = qq.x;
            q[i0][1] = qq.y;
            const float2 hn = fma2(f, before, in);
            h[0] = hn.x; h[1] = hn.y;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float fk = k ? f.y : f.x, ink = k ? in.y : in.x;
            if constexpr (!BACK) {
              if (first[k]) mine[0].b = 0.f;
              mine[0].b = fmaf(fk, mine[0].b, ink);
              mine[0].a *= fk;
            } else {
              if (first[k]) h[0] = 0.f;
              q[i0 + k][0] = (h[0] - x[k]) * (k ? fg.y : fg.x);
              h[0] = fmaf(fk, h[0], ink);
            }
          }
        }
      }
      if constexpr (BACK) {
#pragma unroll
        for (int i = kSeg - 1; i >= 0; --i) {
          float d[V];
          W::open(dh_word(KIND != kAny || i < n, i), d);
          const bool first = MARKS && (KIND == kWhole || KIND == kAny) && ((firsts >> i) & 1u);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float f = gate_f(p[i][v]);
            mine[v].b = first ? 0.f : f * (d[v] + mine[v].b);
            mine[v].a *= f;
          }
        }
      }
    };
    if (kind == kPlain) walk(std::integral_constant<int, kPlain>{});
    else if (MARKS && kind == kMissing) walk(std::integral_constant<int, kMissing>{});
    else if (MARKS && kind == kWhole) walk(std::integral_constant<int, kWhole>{});
    else walk(std::integral_constant<int, kAny>{});
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v].a = MARKS && firsts ? 0.f : fmaxf(mine[v].a, kTiny);
    if (LOAD == kWords) fetch(tile + kBufs * a.ways, buf, (round + kBufs) & 1);  // (this thread has read its words)

    // the maps of the segments before this one: in the warp, then of whole warps
    Map pre[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Map m = mine[v];
      for (int off = lc; off < 32; off <<= 1) {
        const Map up{__shfl_up_sync(0xffffffffu, m.a, off), __shfl_up_sync(0xffffffffu, m.b, off)};
        if (lane >= off) m = after(m, up);
      }
      if (lane >= 32 - lc) s_warp[par][v][warp][col] = m;
      pre[v] = {__shfl_up_sync(0xffffffffu, m.a, lc & 31), __shfl_up_sync(0xffffffffu, m.b, lc & 31)};
      if (lane < lc) pre[v] = {1.f, 0.f};
    }
    // Once a wait has given up the block runs on without waits and arms no barrier, starts no tensor copy and sends nothing
    // more: a barrier whose phase has not ended takes no second arrival.  (Blocks that wait for its maps give up in turn.)
    // Each thread goes by what it knows here: thread 0, which arms the barriers, has waited on all of them.  Leaving the loop
    // by a vote at this barrier cost 8 x 8192 x 2048 bf16 7 % (411 -> 439 us, forward and backward), this nothing (and
    // 1 x 65536 x 4096 f16 forward 2 %, 349 -> 356).
    const bool dead = *(volatile int*)&s_gave_up;
    __syncthreads();
    fetch_side(tile + a.ways);  // (ahead of the barrier it held the block up: 8 x 8192 x 2048 bf16 backward 313 us, here 277)
    if (LOAD == kTensor && !dead) fetch(tile + kBufs * a.ways, buf, (round + kBufs) & 1);

    float s[V];  // the state that reaches this tile, then this segment
    if (a.ways == 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        s[v] = state[v];
        for (int w = 0; w < nwarp; ++w) {
          if (w == warp) s[v] = state[v];
          state[v] = through(s_warp[par][v][w][col], state[v]);
        }
        s[v] = through(pre[v], s[v]);
      }
    } else if (a.cluster) {
      // tell every block of the chain this tile's map, wait for theirs, walk the round's
      const int nch = lc * V;
      if (tid == 0 && !dead) barrier_expect(&s_told[par], (uint32_t)(a.ways * nch) * 8 + a.unsent);
      for (int i = dead ? kMostThreads : tid; i < nch * a.ways; i += nthr) {
        const int ch = i % nch, v = ch / lc, c = ch % lc;
        Map m = tile_map(s_warp[par][v], c, nwarp);
        if (tile >= a.tiles) m = {1.f, 0.f};
        const uint32_t to = (uint32_t)(i / nch);
        send_8(in_block(s_round + (par * kMostCluster + way) * kRowMaps + ch, to), (uint64_t)__float_as_uint(m.b) << 32 | __float_as_uint(m.a),
               in_block(&s_told[par], to));
      }
      if (!dead && !barrier_polls(&s_told[par], (round >> 1) & 1)) wait_more(&s_told[par], (round >> 1) & 1, &s_gave_up, a.tries, a.status);
#pragma unroll
      for (int v = 0; v < V; ++v) {
#pragma unroll 4
        for (int w = 0; w < a.ways; ++w) {
          if (w == way) s[v] = state[v];
          state[v] = through(s_round[(par * kMostCluster + w) * kRowMaps + v * lc + col], state[v]);
        }
        for (int w = 0; w < warp; ++w) s[v] = through(s_warp[par][v][w][col], s[v]);
        s[v] = through(pre[v], s[v]);
      }
    } else {
      // publish the tile's map, wait for the round's, fold them: parts of the round side by side, then in order
      const int nch = lc * V;  // channels of a row
      Map *const s_part = s_round, *const s_pre = s_part + kMostThreads;
      ulonglong2* maps = a.maps + (chain * 2 + par) * (int64_t)a.ways * nch;
      const uint32_t tag = round + 1;
      if (tid < lc) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          Map m = tile_map(s_warp[par][v], col, nwarp);
          if (tile >= a.tiles) m = {1.f, 0.f};
          publish(maps + (int64_t)way * nch + v * lc + col, m, tag + a.unsent);
        }
      }
      // (ways > 1: 256 threads; nch is a power of two up to 64)
      const int ps = 31 - __clz(kMostThreads / nch), parts = 1 << ps, part = tid / nch, ch = tid % nch;
      const int lo = (part * a.ways) >> ps, hi = ((part + 1) * a.ways) >> ps;
      constexpr int kAsk = BACK ? 4 : 2;  // maps in flight (more take registers from the tile: forward 3-8 % slower at 4, both far at 8)
      Map m{1.f, 0.f};
      for (int w0 = lo; w0 < hi; w0 += kAsk) {
        Map k[kAsk];
        uint32_t polls = 0;
        bool all;
        do {
          all = true;
#pragma unroll
          for (int j = 0; j < kAsk; ++j)
            if (w0 + j < hi) all &= published(maps + (int64_t)(w0 + j) * nch + ch, tag, k[j]);
          if (!all && ++polls > a.tries * 1024) {
            *(volatile int*)&s_gave_up = 1;
            if (a.status) atomicOr(a.status, kStatusTimeout);
          }
        } while (!all && !*(volatile int*)&s_gave_up);
#pragma unroll
        for (int j = 0; j < kAsk; ++j) {
          if (w0 + j < hi && w0 + j == way) s_pre[ch] = m;
          if (w0 + j < hi) m = after(k[j], m);
        }
      }
      s_part[part * nch + ch] = m;
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v) {
        for (int k = 0; k < parts; ++k) {
          if (way >= (k * a.ways) >> ps && way < ((k + 1) * a.ways) >> ps) s[v] = through(s_pre[v * lc + col], state[v]);
          state[v] = through(s_part[k * nch + v * lc + col], state[v]);
        }
        for (int w = 0; w < warp; ++w) s[v] = through(s_warp[par][v][w][col], s[v]);
        s[v] = through(pre[v], s[v]);
      }
    }

    // the segment's steps from the state that reaches them
    if (!BACK && n && a.saved) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v == 0 || second) a.saved[(b * nsave + t0 / kSeg) * a.dim + c0 + v] = s[v];
    }
    const auto finish = [&](auto kind_of) {
      constexpr int KIND = decltype(kind_of)::value;
      if constexpr (!BACK) {
        char* const out = py + t0 * a.y.st;
#pragma unroll
        for (int i = 0; i < kSeg; ++i) {
          char* const to = row_of(out, a.y.st, i);
          const bool first = MARKS && (KIND == kWhole || KIND == kAny) && ((firsts >> i) & 1u);
          if constexpr (V == 2) {
            if (first) s[0] = s[1] = 0.f;
            const float2 n2 = fma2(make_float2(p[i][0], p[i][1]), make_float2(s[0], s[1]), make_float2(q[i][0], q[i][1]));
            s[0] = n2.x;
            s[1] = n2.y;
          } else {
            s[0] = fmaf(p[i][0], first ? 0.f : s[0], q[i][0]);
          }
          if (KIND != kAny || i < n) {
            if constexpr (VEC) *reinterpret_cast<uint32_t*>(to) = W::close(s);
            else store_word(to, W::close(s), sizeof(T) == 4 || a.whole, second);
          }
        }
      } else {
        char *const outx = pdx + t0 * a.dx.st, *const outz = pdz + t0 * a.dz.st;
#pragma unroll
        for (int i = kSeg - 1; i >= 0; --i) {
          char *const tx = row_of(outx, a.dx.st, i), *const tz = row_of(outz, a.dz.st, i);
          float d[V], gx[V], gz[V];
          W::open(dh_word(KIND != kAny || i < n, i), d);
          const bool out = KIND != kPlain && MARKS && ((gone >> i) & 1u);
          const bool first = MARKS && (KIND == kWhole || KIND == kAny) && ((firsts >> i) & 1u);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float l = d[v] + s[v];
            gx[v] = out ? 0.f : gate_g(p[i][v]) * l;
            gz[v] = out ? 0.f : q[i][v] * l;
            s[v] = first ? 0.f : gate_f(p[i][v]) * l;
          }
          if (KIND != kAny || i < n) {
            if constexpr (VEC) {
              *reinterpret_cast<uint32_t*>(tx) = W::close(gx);
              *reinterpret_cast<uint32_t*>(tz) = W::close(gz);
            } else {
              store_word(tx, W::close(gx), sizeof(T) == 4 || a.whole, second);
              store_word(tz, W::close(gz), sizeof(T) == 4 || a.whole, second);
            }
          }
        }
      }
    };
    if (n) {
      if (kind == kPlain || (!BACK && kind == kMissing)) finish(std::integral_constant<int, kPlain>{});
      else if (MARKS && kind == kMissing) finish(std::integral_constant<int, kMissing>{});
      else if (MARKS && kind == kWhole) finish(std::integral_constant<int, kWhole>{});
      else finish(std::integral_constant<int, kAny>{});
      if (a.end && (BACK ? t0 == 0 : t0 + n == a.time)) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v == 0 || second) a.end[b * a.dim + c0 + v] = s[v];
      }
    }
  }
  // after a wait that gave up, copies in flight end before their memory is given back
  if (LOAD == kWords) copies_done<0>();
  if (LOAD == kTensor) {
    __syncthreads();
    if (s_gave_up) {
      const unsigned long long until = device_ns() + 20000000ull;
      while (device_ns() < until) {}
    }
  }
  if (a.cluster) cluster_sync();  // (no block ends while another may still write to it)
}

// How a call's work is laid out: by its sizes and type alone, so that strides and alignment change no bit.
struct Plan {
  int lc, threads, ways, groups;
  bool cluster;
  int64_t chains, tiles;
  uint64_t map_bytes;
};

int sm_count(int* out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev);
  return (int)e;
}

mf_status plan_of(int type, int64_t batch, int64_t time, int64_t dim, bool back, Plan* out) {
  const int V = type == MF_TYPE_F32 ? 1 : 2;
  Plan p{};
  const int64_t words = (dim + V - 1) / V;
  p.lc = 1;
  while (p.lc < 32 && p.lc < words) p.lc *= 2;
  const int64_t segs = (time + kSeg - 1) / kSeg;
  p.threads = 32;
  while (p.threads < kMostThreads && p.threads / p.lc < segs) p.threads *= 2;
  p.groups = (int)((words + p.lc - 1) / p.lc);
  p.chains = batch * p.groups;
  if (p.chains > 0x7FFFFFFF) {  // (a block each, and more only where there are few)
    set_error("mf_recurrence: too many sequences of these channels for a launch");
    return MF_EINVAL;
  }
  p.tiles = (segs + p.threads / p.lc - 1) / (p.threads / p.lc);
  p.ways = 1;
  if (p.tiles > 1) {
    int sms = 0;
    const cudaError_t e = (cudaError_t)sm_count(&sms);
    if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute");
    const int per_sm = type == MF_TYPE_F32 ? (back ? blocks_per_sm<float, true>() : blocks_per_sm<float, false>())
                                           : (back ? blocks_per_sm<__half, true>() : blocks_per_sm<__half, false>());
    const int64_t slots = (int64_t)sms * per_sm;
    // Where a chain has so many blocks that a thread would fold more than 20 of their maps (a round trip each few), narrower
    // rows, down to a sector: more chains of fewer blocks each, and more threads a map.  Forward, wide rows -> narrow: bf16
    // 1 x 262144 x 40 142 -> 54 us, 1 x 65536 x 40 48 -> 25, 1 x 65536 x 128 56 -> 37, 1 x 20000 x 100 33 -> 17; f32 1 x 262144 x
    // 16 62 -> 37, 1 x 100000 x 64 50 -> 39, 1 x 1000000 x 32 300 -> 158.  Below that rows of 32 words, which tensor copies read,
    // are as fast or faster (f32 2 x 100000 x 100 84 against 97, backward 115 against 140; 4 x 65536 x 32 44 against 46, 48 against
    // 58).  Of 13 shapes none was slower than the better of both by more than 5 %.
    for (int64_t most = 20; p.lc > 8; most = 4) {
      const int64_t ways = slots / p.chains < p.tiles ? slots / p.chains : p.tiles;
      if (ways < 2 * kMostCluster || ways * p.lc * V <= most * kMostThreads) break;
      p.lc /= 2;
      p.groups = (int)((words + p.lc - 1) / p.lc);
      p.chains = batch * p.groups;
      p.tiles = (segs + p.threads / p.lc - 1) / (p.threads / p.lc);
    }
    const int64_t all = slots / p.chains;  // blocks a chain could have
    int64_t ways = 1;
    while (ways < kMostCluster && 2 * ways <= all && 2 * ways <= p.tiles) ways *= 2;
    p.cluster = ways > 1;
    // more blocks than a cluster's where there is room for twice as many and work for them
    const int64_t most = all < p.tiles ? all : p.tiles;
    if (most >= 2 * kMostCluster) {
      ways = most;
      p.cluster = false;
    }
    p.ways = (int)ways;
  }
  if (p.ways > 1 && !p.cluster) {
    p.map_bytes = (uint64_t)p.chains * 2 * p.ways * p.lc * V * sizeof(ulonglong2);
  }
  *out = p;
  return MF_OK;
}

template <typename T, bool BACK, int LOAD, bool MARKS>
mf_status launch(Args& a, Maps3& maps, const Plan& p, cudaStream_t s) {
  const auto kernel = k_recur<T, BACK, LOAD, MARKS>;
  const size_t smem = LOAD == kDirect ? 0 : (size_t)(2 * buffers<T, BACK>() + (BACK ? 2 : 0)) * kSeg * kMostThreads * 4 + 128;
  if (smem) MF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  if (p.ways == 1) {
    kernel<<<(unsigned)p.chains, p.threads, smem, s>>>(a, maps);
    MF_CUDA(cudaGetLastError());
    return MF_OK;
  }
  if (p.cluster) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.chains * p.ways));
    cfg.blockDim = dim3(p.threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)p.ways;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    MF_CUDA(cudaLaunchKernelEx(&cfg, kernel, a, maps));
    return MF_OK;
  }
  void* args[] = {&a, &maps};
  MF_CUDA(cudaLaunchCooperativeKernel((const void*)kernel, dim3((unsigned)(p.chains * p.ways)), dim3(p.threads), args, smem, s));
  return MF_OK;
}

template <typename T, bool BACK>
mf_status launch_of(Args& a, Maps3& maps, const Plan& p, int load, cudaStream_t s) {
  if (load == kTensor) return a.marks ? launch<T, BACK, kTensor, true>(a, maps, p, s) : launch<T, BACK, kTensor, false>(a, maps, p, s);
  if (load == kWords) return a.marks ? launch<T, BACK, kWords, true>(a, maps, p, s) : launch<T, BACK, kWords, false>(a, maps, p, s);
  return a.marks ? launch<T, BACK, kDirect, true>(a, maps, p, s) : launch<T, BACK, kDirect, false>(a, maps, p, s);
}

bool whole_words(const Seq& t, int64_t batch, int64_t time) {
  return ((uintptr_t)t.p & 3) == 0 && (batch < 2 || (t.sb & 3) == 0) && (time < 2 || (t.st & 3) == 0);
}

// The map of a [batch][time][dim] tensor with a box of `steps` rows of 32 words; false where tensor copies cannot read it.
bool map_of(CUtensorMap* map, const Seq& t, int type, int64_t batch, int64_t time, int64_t dim, int steps) {
  const int64_t size = type == MF_TYPE_F32 ? 4 : 2, row = (dim * size + 15) / 16 * 16;
  const int64_t st = time < 2 ? row : t.st, sb = batch < 2 ? row : t.sb;
  if (((uintptr_t)t.p & 15) || st % 16 || sb % 16 || st <= 0 || sb <= 0 || st >= (int64_t(1) << 40) || sb >= (int64_t(1) << 40)) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)time, (cuuint64_t)batch}, strides[2] = {(cuuint64_t)st, (cuuint64_t)sb};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / size), (cuuint32_t)steps, 1};
  return tensor_map(map, type == MF_TYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == MF_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                                                     : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                    3, t.p, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <bool BACK>
mf_status run(Args& a, int type, void* work, uint32_t wait_test, cudaStream_t s) {
  const size_t state = sizeof(float) * (size_t)(a.batch * a.dim);
  if (a.time == 0) {
    if (!a.end) return MF_OK;
    if (a.first) MF_CUDA(cudaMemcpyAsync(a.end, a.first, state, cudaMemcpyDeviceToDevice, s));
    else MF_CUDA(cudaMemsetAsync(a.end, 0, state, s));
    return MF_OK;
  }
  Plan p;
  const mf_status st = plan_of(type, a.batch, a.time, a.dim, BACK, &p);
  if (st != MF_OK) return st;
  a.tiles = p.tiles;
  a.groups = p.groups;
  a.lc = p.lc;
  a.ways = p.ways;
  a.cluster = p.cluster;
  a.tries = wait_test ? wait_test : kTries;
  a.unsent = wait_test ? 16 : 0;
  if (p.ways > 1 && !p.cluster) {
    a.maps = (ulonglong2*)work;
    MF_CUDA(cudaMemsetAsync(work, 0, p.map_bytes, s));  // (no tag is 0)
  }
  const int64_t b = a.batch, t = a.time;
  a.whole = type == MF_TYPE_F32 || (a.dim % 2 == 0 && whole_words(a.x, b, t) && whole_words(a.z, b, t) && whole_words(a.y, b, t) &&
                   (!BACK || (whole_words(a.dx, b, t) && whole_words(a.dz, b, t))));
  a.marks16 = a.marks && a.mt == 1 && ((uintptr_t)a.marks & 15) == 0 && (b < 2 || (a.mb & 15) == 0);
  Maps3 maps;
  const int steps = p.threads / p.lc * kSeg;
  int load = p.threads < kMostThreads || !a.whole ? kDirect : kWords;
  if (load == kWords && p.lc == 32 && map_of(&maps.x, a.x, type, b, t, a.dim, steps) && map_of(&maps.z, a.z, type, b, t, a.dim, steps) &&
      (!BACK || map_of(&maps.y, a.y, type, b, t, a.dim, steps)))
    load = kTensor;
  if (type == MF_TYPE_F32) return launch_of<float, BACK>(a, maps, p, load, s);
  if (type == MF_TYPE_BF16) return launch_of<__nv_bfloat16, BACK>(a, maps, p, load, s);
  return launch_of<__half, BACK>(a, maps, p, load, s);
}

Seq seq(const mf_seq& t, int type) {
  const int64_t size = type == MF_TYPE_F32 ? 4 : 2;
  return {(char*)t.d_ptr, t.stride_batch * size, t.stride_time * size};
}

}  // namespace

mf_status recur_work(int type, int64_t batch, int64_t time, int64_t dim, bool backward, uint64_t* bytes) {
  *bytes = 0;
  if (!batch || !time || !dim) return MF_OK;
  Plan p;
  const mf_status st = plan_of(type, batch, time, dim, backward, &p);
  if (st == MF_OK) *bytes = p.map_bytes;
  return st;
}

mf_status recur_forward(const mf_recurrence_args& p, void* work, uint32_t wait_test, cudaStream_t s) {
  Args a{};
  a.batch = p.batch; a.time = p.time; a.dim = p.dim;
  a.x = seq(p.x, p.type); a.z = seq(p.z, p.type); a.y = seq(p.h, p.type);
  a.marks = p.d_marks; a.mb = p.marks_stride_batch; a.mt = p.marks_stride_time;
  a.first = p.d_h0; a.end = p.d_last; a.saved = p.d_saved; a.status = p.d_status;
  return run<false>(a, p.type, work, wait_test, s);
}

mf_status recur_backward(const mf_recurrence_grad_args& p, void* work, uint32_t wait_test, cudaStream_t s) {
  Args a{};
  a.batch = p.batch; a.time = p.time; a.dim = p.dim;
  a.x = seq(p.x, p.type); a.z = seq(p.z, p.type); a.y = seq(p.dh, p.type);
  a.dx = seq(p.dx, p.type); a.dz = seq(p.dz, p.type);
  a.marks = p.d_marks; a.mb = p.marks_stride_batch; a.mt = p.marks_stride_time;
  a.saved = const_cast<float*>(p.d_saved);
  a.first = p.d_dlast; a.end = p.d_dh0; a.status = p.d_status;
  return run<true>(a, p.type, work, wait_test, s);
}

}  // namespace mf
