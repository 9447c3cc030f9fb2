// Gated linear recurrence over sequences and its gradient (the operators' section of include/mf.h).
//
// h_t = f_t h_{t-1} + g_t x_t is a chain of maps s -> A s + B, and maps compose: (A2, B2) after (A1, B1) is
// (A2 A1, A2 B1 + B2).  The gradient is such a chain too, from the last step to the first, on the value b
// that a step passes back: b <- f_t (dh_t + b).  Both kernels below are one pass over the data:
//
//   a thread holds one 32-bit word (one fp32 channel, or two 16-bit ones) of 16 steps in registers;
//   the lanes of a row of `lc` words (32 where there are as many) lie side by side, so a warp reads and writes whole
//   sectors;
//   a block of up to 256 threads holds a tile of (256 / lc) segments of 16 steps, scans the segments'
//   maps (shuffles within a warp, shared memory between warps), and then walks its 16 steps with the
//   state that reaches them.
//
// A chain (a batch row's group of lc words) is walked tile after tile by one block where there are chains
// enough to fill the GPU.  Else `ways` blocks share it: in each round they take neighbouring tiles, publish
// their tiles' maps, wait for the others' (all blocks are resident: a cooperative launch) and fold the maps
// of the round in a fixed order, so equal calls give equal bits.  The next tile's words are copied to
// shared memory before the wait: rows of 32 words by one tensor copy (TMA) a tensor, narrower ones by cp.async; rows
// that do not start and end on words are read without.
//
// Bound: memory, 3 words read and written per word of x forward, 5 backward (x and z again, since the rest
// of a network ran between); the backward call starts each segment from the state that the forward call
// saved for it (4 bytes for 16 steps of a channel), so it needs h neither in memory nor rounded.
#include <type_traits>

#include "mf_ops.cuh"
#include "tma.cuh"

namespace mf {
namespace {

constexpr int kSeg = kRecurSave;   // steps of a thread
constexpr int kMostThreads = 256;
constexpr float kTiny = 1e-37f;    // least factor of a map that cuts nothing (see Map)
constexpr uint32_t kPolls = 1u << 22;  // of a bounded wait, each an L2 round trip (seconds in all)

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
  int64_t tiles;
  int groups, lc, ways;
};

// s -> a s + b.  a is 0 only where a first sample cuts the chain, and then nothing of s passes, not even a
// NaN or an infinity; products of factors that underflow stay at kTiny (times a state: nothing) so that they do not cut.
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
  static __device__ __forceinline__ void open(uint32_t w, float (&v)[1]) { v[0] = __uint_as_float(w); }
  static __device__ __forceinline__ uint32_t close(const float (&v)[1]) { return __float_as_uint(v[0]); }
};
template <> struct Words<__nv_bfloat16> {
  static constexpr int V = 2;
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
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// A word of two 16-bit channels whose address may be odd, or whose second channel may not exist.
__device__ __forceinline__ uint32_t load_halves(const char* p, bool second) {
  const uint32_t lo = *reinterpret_cast<const uint16_t*>(p);
  return second ? lo | ((uint32_t)*reinterpret_cast<const uint16_t*>(p + 2) << 16) : lo;
}
__device__ __forceinline__ void store_halves(char* p, uint32_t w, bool second) {
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

// Blocks of an SM.  Forward, 16-bit: 64 registers of (f, g x) a thread; backward 80 (gate, dz / l, dh).
template <typename T, bool BACK> constexpr int blocks_per_sm() { return sizeof(T) == 4 ? (BACK ? 2 : 3) : 2; }

// How a tile's words come in.  kTensor: rows of 32 words by tensor copies (rows on 16 bytes).  kWords: every row starts
// on a word and ends with one, so that words are copied whole.  kHalves: 16-bit loads.
enum Load { kTensor, kWords, kHalves };

struct Maps3 {
  CUtensorMap x, z, y;
};

template <typename T, bool BACK, int LOAD, bool MARKS>
__global__ void __launch_bounds__(kMostThreads, blocks_per_sm<T, BACK>()) k_recur(const Args a, const __grid_constant__ Maps3 maps3) {
  constexpr bool VEC = LOAD != kHalves;
  constexpr int kTileWords = kSeg * kMostThreads;       // of one tensor in shared memory
  using W = Words<T>;
  constexpr int V = W::V;
  // kTensor: [tensor][step of the tile][32]; kWords: [tensor][step of the segment][thread]
  extern __shared__ uint32_t s_raw[];
  uint32_t* const s_words = s_raw + ((128 - (shared_u32(s_raw) & 127)) & 127) / 4;  // (tensor copies write from 128 bytes on)
  __shared__ uint64_t s_bar;
  __shared__ Map s_warp[2][V][kMostThreads / 32][32];   // [tile parity]: maps of the warps' segments
  __shared__ Map s_part[V][kMostThreads], s_pre[V][32];  // (ways > 1) maps of parts of a round, and of what precedes the tile
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
  if (tid == 0) s_gave_up = 0;
  if constexpr (LOAD == kTensor) {
    if (tid == 0) {
      barrier_init(&s_bar, 1);
      barrier_init_fence();
    }
    __syncthreads();
  }
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
  uint32_t marks[4], saved_w[V];
  // what a tile needs from memory: its words to shared memory, its marks and saved states to registers
  auto fetch = [&](int64_t tile) {
    int64_t t0;
    const int n = segment(tile, t0);
    if constexpr (LOAD == kTensor) {  // (every thread has read its words of the tile before)
      if (tid == 0) {
        const int32_t e0 = (int32_t)(chain % a.groups) * 32 * V, e2 = (int32_t)b;
        const int32_t e1 = (int32_t)((BACK ? a.tiles - 1 - tile : tile) * nseg * kSeg);
        barrier_expect(&s_bar, (BACK ? 3 : 2) * (uint32_t)nthr * kSeg * 4);
        tma_load_3d(s_words, &maps3.x, e0, e1, e2, &s_bar);
        tma_load_3d(s_words + kTileWords, &maps3.z, e0, e1, e2, &s_bar);
        if constexpr (BACK) tma_load_3d(s_words + 2 * kTileWords, &maps3.y, e0, e1, e2, &s_bar);
      }
    }
    if constexpr (LOAD == kWords) {
      if (n) {
        const char *qx = px + t0 * a.x.st, *qz = pz + t0 * a.z.st, *qy = BACK ? py + t0 * a.y.st : nullptr;
        uint32_t* to = s_words + tid;
#pragma unroll
        for (int i = 0; i < kSeg; ++i) {
          if (i < n) {
            copy_word(to + i * kMostThreads, qx);
            copy_word(to + kTileWords + i * kMostThreads, qz);
            if constexpr (BACK) copy_word(to + 2 * kTileWords + i * kMostThreads, qy);
          }
          qx += a.x.st;
          qz += a.z.st;
          if constexpr (BACK) qy += a.y.st;
        }
      }
    }
    if constexpr (MARKS) {
      marks[0] = marks[1] = marks[2] = marks[3] = 0;
      if (n) {
        const uint8_t* pm = a.marks + b * a.mb + t0 * a.mt;
        if (n == kSeg && a.marks16) {
          const uint4 w = *reinterpret_cast<const uint4*>(pm);
          marks[0] = w.x; marks[1] = w.y; marks[2] = w.z; marks[3] = w.w;
        } else {
          for (int i = 0; i < n; ++i) {
            const uint32_t m = (uint32_t)pm[i * a.mt] << (8 * (i & 3));
            if (i < 4) marks[0] |= m; else if (i < 8) marks[1] |= m; else if (i < 12) marks[2] |= m; else marks[3] |= m;
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
  if (tile < a.tiles) fetch(tile);
  for (uint32_t round = 0; (int64_t)round * a.ways < a.tiles; ++round, tile += a.ways) {
    int64_t t0;
    const int n = tile < a.tiles ? segment(tile, t0) : 0;
    // forward: p = f, q = g x.  backward: p = the gate, q = dz / l, r = dh's words.  Steps that are not there: f = 1, q = 0.
    float p[kSeg][V], q[kSeg][V];
    uint32_t r[kSeg];
    uint32_t firsts = 0, gone = 0;  // bits of the segment's steps
    if constexpr (LOAD == kWords) copies_done();
    if constexpr (LOAD == kTensor) {
      if (tile < a.tiles && !barrier_wait(&s_bar, round & 1) && a.status) atomicOr(a.status, kStatusTimeout);
    }
    if constexpr (MARKS) {
#pragma unroll
      for (int i = 0; i < kSeg; ++i) {
        const uint32_t m = (marks[i / 4] >> (8 * (i & 3))) & 0xFFu;
        firsts |= (m == MF_MARK_FIRST ? 1u : 0u) << i;
        gone |= (m == MF_MARK_MISSING ? 1u : 0u) << i;
      }
    }
    gone |= ~0u << n;
    // where all of a warp's steps are samples, without conditions
    const bool plain = VEC && __all_sync(0xffffffffu, (gone & ((1u << kSeg) - 1)) == 0 && firsts == 0);
    Map mine[V];
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      mine[v] = {1.f, 0.f};
      h[v] = BACK ? __uint_as_float(saved_w[v]) : 0.f;
    }
    const auto walk = [&](auto is_plain) {
      constexpr bool PLAIN = decltype(is_plain)::value;
      [[maybe_unused]] const char *qx = px, *qz = pz, *qy = py;
      if constexpr (!VEC) {
        if (n) {
          qx += t0 * a.x.st;
          qz += t0 * a.z.st;
          if constexpr (BACK) qy += t0 * a.y.st;
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
          r[i] = 0;
          if (PLAIN || i < n) {
            if constexpr (VEC) {
              wx = mine_w[i * kStep];
              wz = mine_w[kTileWords + i * kStep];
              if constexpr (BACK) r[i] = mine_w[2 * kTileWords + i * kStep];
            } else {
              wx = load_halves(qx, second);
              wz = load_halves(qz, second);
              if constexpr (BACK) r[i] = load_halves(qy, second);
            }
          }
          if constexpr (!VEC) {
            qx += a.x.st;
            qz += a.z.st;
            if constexpr (BACK) qy += a.y.st;
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
        const float2 in2 = mul2(g, make_float2(x[0], x[1]));
        const float2 f2 = make_float2(z[0] < 0.f ? small.x : large.x, z[1] < 0.f ? small.y : large.y);
        if constexpr (PLAIN && V == 2) {
          if constexpr (!BACK) {
            p[i0][0] = f2.x; p[i0][1] = f2.y;
            q[i0][0] = in2.x; q[i0][1] = in2.y;
            const float2 mb = fma2(f2, make_float2(mine[0].b, mine[1].b), in2), ma = mul2(f2, make_float2(mine[0].a, mine[1].a));
            mine[0] = {ma.x, mb.x};
            mine[1] = {ma.y, mb.y};
          } else {
            p[i0][0] = pack_gate(small.x, z[0]); p[i0][1] = pack_gate(small.y, z[1]);
            const float2 h2 = make_float2(h[0], h[1]);
            const float2 qq = mul2(add2(h2, make_float2(-x[0], -x[1])), fg);
            q[i0][0] = qq.x; q[i0][1] = qq.y;
            const float2 hn = fma2(f2, h2, in2);
            h[0] = hn.x; h[1] = hn.y;
          }
        } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int i = i0 + k / V, v = k % V;
          float f = k ? f2.y : f2.x, in = k ? in2.y : in2.x;
          const bool out = !PLAIN && ((gone >> i) & 1u), first = !PLAIN && MARKS && ((firsts >> i) & 1u);
          if (out) { f = 1.f; in = 0.f; }
          if constexpr (!BACK) {
            if (first) f = 0.f;
            p[i][v] = f;
            q[i][v] = in;
            mine[v].b = first ? in : fmaf(f, mine[v].b, in);
            mine[v].a *= f;
          } else {
            const float before = first ? 0.f : h[v];
            p[i][v] = out ? 0.f : pack_gate(k ? small.y : small.x, z[k]);
            q[i][v] = out ? 0.f : (before - x[k]) * (k ? fg.y : fg.x);
            h[v] = first ? in : fmaf(f, h[v], in);
          }
        }
        }
      }
      if constexpr (BACK) {
#pragma unroll
        for (int i = kSeg - 1; i >= 0; --i) {
          float d[V];
          W::open(r[i], d);
          const bool first = !PLAIN && MARKS && ((firsts >> i) & 1u);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float f = gate_f(p[i][v]);
            mine[v].b = first ? 0.f : f * (d[v] + mine[v].b);
            mine[v].a *= f;
          }
        }
      }
    };
    if (plain) walk(std::true_type{});
    else walk(std::false_type{});
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v].a = MARKS && firsts ? 0.f : fmaxf(mine[v].a, kTiny);
    if (LOAD != kTensor && tile + a.ways < a.tiles) fetch(tile + a.ways);  // (this thread has read its words)

    // the maps of the segments before this one: in the warp, then of whole warps
    Map pre[V];
    const int par = round & 1;
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
    __syncthreads();
    if (LOAD == kTensor && tile + a.ways < a.tiles) fetch(tile + a.ways);

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
    } else {
      // publish the tile's map, wait for the round's, fold them: parts of the round side by side, then in order
      const int nch = lc * V;  // channels of a row
      ulonglong2* maps = a.maps + (chain * 2 + par) * (int64_t)a.ways * nch;
      const uint32_t tag = round + 1;
      if (tid < lc) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          Map m = s_warp[par][v][0][col];
          for (int w = 1; w < nwarp; ++w) m = after(s_warp[par][v][w][col], m);
          if (tile >= a.tiles) m = {1.f, 0.f};
          publish(maps + (int64_t)way * nch + v * lc + col, m, tag);
        }
      }
      // (ways > 1: 256 threads; nch is a power of two up to 64)
      const int ps = 31 - __clz(kMostThreads / nch), parts = 1 << ps, part = tid / nch, ch = tid % nch;
      const int lo = (part * a.ways) >> ps, hi = ((part + 1) * a.ways) >> ps;
      Map m{1.f, 0.f};
      for (int w0 = lo; w0 < hi; w0 += 4) {
        Map k[4];
        uint32_t polls = 0;
        bool all;
        do {  // (four words in flight)
          all = true;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (w0 + j < hi) all &= published(maps + (int64_t)(w0 + j) * nch + ch, tag, k[j]);
          if (!all && ++polls > kPolls) {
            *(volatile int*)&s_gave_up = 1;
            if (a.status) atomicOr(a.status, kStatusTimeout);
          }
        } while (!all && !*(volatile int*)&s_gave_up);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (w0 + j < hi && w0 + j == way) s_pre[ch / lc][ch % lc] = m;
          if (w0 + j < hi) m = after(k[j], m);
        }
      }
      s_part[ch / lc][part * lc + ch % lc] = m;
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v) {
        for (int k = 0; k < parts; ++k) {
          if (way >= (k * a.ways) >> ps && way < ((k + 1) * a.ways) >> ps) s[v] = through(s_pre[v][col], state[v]);
          state[v] = through(s_part[v][k * lc + col], state[v]);
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
    const auto finish = [&](auto is_plain) {
      constexpr bool PLAIN = decltype(is_plain)::value;
      if constexpr (!BACK) {
        char* const out = py + t0 * a.y.st;
#pragma unroll
        for (int i = 0; i < kSeg; ++i) {
          char* const to = row_of(out, a.y.st, i);
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (!(PLAIN && V == 2)) s[v] = !PLAIN && MARKS && ((firsts >> i) & 1u) ? q[i][v] : fmaf(p[i][v], s[v], q[i][v]);
          if constexpr (PLAIN && V == 2) {
            const float2 n2 = fma2(make_float2(p[i][0], p[i][1]), make_float2(s[0], s[1]), make_float2(q[i][0], q[i][1]));
            s[0] = n2.x;
            s[1] = n2.y;
          }
          if (PLAIN || i < n) {
            if constexpr (VEC) *reinterpret_cast<uint32_t*>(to) = W::close(s);
            else store_halves(to, W::close(s), second);
          }
        }
      } else {
        char *const outx = pdx + t0 * a.dx.st, *const outz = pdz + t0 * a.dz.st;
#pragma unroll
        for (int i = kSeg - 1; i >= 0; --i) {
          char *const tx = row_of(outx, a.dx.st, i), *const tz = row_of(outz, a.dz.st, i);
          float d[V], gx[V], gz[V];
          W::open(r[i], d);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float l = d[v] + s[v];
            const bool out = !PLAIN && MARKS && ((gone >> i) & 1u);
            gx[v] = out ? 0.f : gate_g(p[i][v]) * l;
            gz[v] = out ? 0.f : q[i][v] * l;
            s[v] = !PLAIN && MARKS && ((firsts >> i) & 1u) ? 0.f : gate_f(p[i][v]) * l;
          }
          if (PLAIN || i < n) {
            if constexpr (VEC) {
              *reinterpret_cast<uint32_t*>(tx) = W::close(gx);
              *reinterpret_cast<uint32_t*>(tz) = W::close(gz);
            } else {
              store_halves(tx, W::close(gx), second);
              store_halves(tz, W::close(gz), second);
            }
          }
        }
      }
    };
    if (n) {
      if (plain) finish(std::true_type{});
      else finish(std::false_type{});
      if (a.end && (BACK ? t0 == 0 : t0 + n == a.time)) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v == 0 || second) a.end[b * a.dim + c0 + v] = s[v];
      }
    }
  }
}

// How a call's work is laid out: by its sizes and type alone, so that strides and alignment change no bit.
struct Plan {
  int lc, threads, ways, groups;
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
  p.tiles = (segs + p.threads / p.lc - 1) / (p.threads / p.lc);
  p.ways = 1;
  if (p.tiles > 1) {
    int sms = 0;
    const cudaError_t e = (cudaError_t)sm_count(&sms);
    if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute");
    const int per_sm = type == MF_TYPE_F32 ? (back ? blocks_per_sm<float, true>() : blocks_per_sm<float, false>())
                                           : (back ? blocks_per_sm<__half, true>() : blocks_per_sm<__half, false>());
    const int64_t ways = (int64_t)sms * per_sm / p.chains;
    p.ways = (int)(ways < 1 ? 1 : ways < p.tiles ? ways : p.tiles);
  }
  if (p.ways > 1) {
    p.map_bytes = (uint64_t)p.chains * 2 * p.ways * p.lc * V * sizeof(ulonglong2);
  }
  *out = p;
  return MF_OK;
}

template <typename T, bool BACK, int LOAD, bool MARKS>
mf_status launch(Args& a, Maps3& maps, const Plan& p, cudaStream_t s) {
  const auto kernel = k_recur<T, BACK, LOAD, MARKS>;
  const size_t smem = LOAD == kHalves ? 0 : (size_t)(BACK ? 3 : 2) * kSeg * kMostThreads * 4 + 128;
  MF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  if (p.ways == 1) {
    kernel<<<(unsigned)p.chains, p.threads, smem, s>>>(a, maps);
    MF_CUDA(cudaGetLastError());
    return MF_OK;
  }
  void* args[] = {&a, &maps};
  MF_CUDA(cudaLaunchCooperativeKernel((const void*)kernel, dim3((unsigned)(p.chains * p.ways)), dim3(p.threads), args, smem, s));
  return MF_OK;
}

template <typename T, bool BACK>
mf_status launch_of(Args& a, Maps3& maps, const Plan& p, int load, cudaStream_t s) {
  if (load == kTensor) return a.marks ? launch<T, BACK, kTensor, true>(a, maps, p, s) : launch<T, BACK, kTensor, false>(a, maps, p, s);
  if constexpr (sizeof(T) == 2) {
    if (load == kHalves)
      return a.marks ? launch<T, BACK, kHalves, true>(a, maps, p, s) : launch<T, BACK, kHalves, false>(a, maps, p, s);
  }
  return a.marks ? launch<T, BACK, kWords, true>(a, maps, p, s) : launch<T, BACK, kWords, false>(a, maps, p, s);
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
mf_status run(Args& a, int type, void* work, cudaStream_t s) {
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
  if (p.ways > 1) {
    a.maps = (ulonglong2*)work;
    MF_CUDA(cudaMemsetAsync(work, 0, p.map_bytes, s));  // (no tag is 0)
  }
  const int64_t b = a.batch, t = a.time;
  const bool vec = a.dim % 2 == 0 && whole_words(a.x, b, t) && whole_words(a.z, b, t) && whole_words(a.y, b, t) &&
                   (!BACK || (whole_words(a.dx, b, t) && whole_words(a.dz, b, t)));
  a.marks16 = a.marks && a.mt == 1 && ((uintptr_t)a.marks & 15) == 0 && (b < 2 || (a.mb & 15) == 0);
  Maps3 maps;
  const int steps = p.threads / p.lc * kSeg;
  int load = type != MF_TYPE_F32 && !vec ? kHalves : kWords;
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

mf_status recur_forward(const mf_recurrence_args& p, void* work, cudaStream_t s) {
  Args a{};
  a.batch = p.batch; a.time = p.time; a.dim = p.dim;
  a.x = seq(p.x, p.type); a.z = seq(p.z, p.type); a.y = seq(p.h, p.type);
  a.marks = p.d_marks; a.mb = p.marks_stride_batch; a.mt = p.marks_stride_time;
  a.first = p.d_h0; a.end = p.d_last; a.saved = p.d_saved; a.status = p.d_status;
  return run<false>(a, p.type, work, s);
}

mf_status recur_backward(const mf_recurrence_grad_args& p, void* work, cudaStream_t s) {
  Args a{};
  a.batch = p.batch; a.time = p.time; a.dim = p.dim;
  a.x = seq(p.x, p.type); a.z = seq(p.z, p.type); a.y = seq(p.dh, p.type);
  a.dx = seq(p.dx, p.type); a.dz = seq(p.dz, p.type);
  a.marks = p.d_marks; a.mb = p.marks_stride_batch; a.mt = p.marks_stride_time;
  a.saved = const_cast<float*>(p.d_saved);
  a.first = p.d_dlast; a.end = p.d_dh0; a.status = p.d_status;
  return run<true>(a, p.type, work, s);
}

}  // namespace mf
