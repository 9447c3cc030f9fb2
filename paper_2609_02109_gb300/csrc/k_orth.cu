// Orthogonalisation of matrices by Newton-Schulz products (the operators' section of include/mf.h).
//
// Each matrix is worked on as X [m][n] with m <= n (a tall one as its transpose: the polynomial is the same).  A step is
// three products: A = X X^T, B = b A + c A A, X' = a X + B X.  A and B are symmetric, so only tiles that reach the
// diagonal or lie below it are computed, and written to both sides.
//
// Operands are fp16 numbers scaled by powers of two: one part (11 bits) or two (hi + lo, 22 bits; the product is then
// hi hi + hi lo + lo hi).  A product P Q^T reads both operands along rows, so X is kept as X and as X^T (the epilogue of
// X' writes both; 2 or 4 bytes an element more, against a second way to lay operands out).
#include <atomic>
#include <cmath>

#include "mf_ops.cuh"
#include "tma.cuh"

namespace mf {
namespace {

// ------------------------------------------------------------------------------------------
// The norm and the first operands
// ------------------------------------------------------------------------------------------

// A matrix's squares in three ranges, so that none overflows or underflows in fp32: small values scaled by 2^96,
// large ones by 2^-90.  No sum of 2^40 squares, the most that a matrix has, passes 2^120.
struct Squares {
  float mid = 0.f, small = 0.f, large = 0.f;
  __device__ __forceinline__ void add(float v) {
    const float m = fabsf(v);
    if (m < 0x1p-62f) small = fmaf(v * 0x1p96f, v * 0x1p96f, small);
    else if (m > 0x1p40f) large = fmaf(v * 0x1p-90f, v * 0x1p-90f, large);
    else mid = fmaf(v, v, mid);  // (NaN too)
  }
  __device__ __forceinline__ void add(const Squares& q) {
    mid += q.mid;
    small += q.small;
    large += q.large;
  }
};
__device__ __forceinline__ Squares warp_sum(Squares q) {
  for (int w = 16; w > 0; w >>= 1) {
    q.mid += __shfl_xor_sync(0xffffffffu, q.mid, w);
    q.small += __shfl_xor_sync(0xffffffffu, q.small, w);
    q.large += __shfl_xor_sync(0xffffffffu, q.large, w);
  }
  return q;
}

// What a matrix's values are multiplied by to become operands, s0 s1 (two powers of two, each a normal number), and the
// factor that makes the operands X: X = operand * rho.  The norm of the operands lies in [2^12, 2^13), so
// no value leaves fp16's range, and 16-bit values become operands without a rounding.
struct Scale {
  float s0, s1, rho;
  float norm;  // of X: below 1 by what eps adds
};
__device__ __forceinline__ Scale scale_of(const Squares& q, float eps) {
  // the sum of squares as base 2^shift (what is left out is below 2^-30 of it)
  float base = q.mid;
  int shift = 0;
  if (q.large > 0.f) {
    base = fmaf(q.mid * 0x1p-90f, 0x1p-90f, q.large);
    shift = 180;
  } else if (q.mid < 0x1p-70f) {
    base = fmaf(q.mid * 0x1p96f, 0x1p96f, q.small);
    shift = -192;
  }
  if (base == 0.f) return {1.f, 1.f, 0.f, 0.f};  // (zeros stay zeros)
  if (!isfinite(q.mid + q.large)) return {1.f, 1.f, __int_as_float(0x7fc00000), 1.f};
  const float n = sqrtf(base);
  int e;
  frexpf(n, &e);  // the norm is n 2^(shift / 2), n = f 2^e, f in [1/2, 1)
  const int k = 13 - e - shift / 2;
  const float scaled = ldexpf(n, 13 - e), more = ldexpf(eps, k);
  const float rho = isfinite(more) ? 1.f / (scaled + more) : ldexpf(1.f / eps, -k);
  return {ldexpf(1.f, k / 2), ldexpf(1.f, k - k / 2), rho, scaled * rho};
}

// A step's factors (steps_of): result = acc * sum + old * old.
struct Factors {
  float gram, square_acc, square_old, apply_acc, apply_old;
};
struct Step {
  Factors f;
  float top;              // no singular value of the X that it starts from is larger
  int parts, next_parts;  // of its operands A and B, and of the X that it makes
};
struct Steps {
  int n;
  float a, b, c;
  Step step[MF_ORTH_MAX_STEPS];
};

// The exponent of the power of two that operands whose largest singular value is at most `top` are multiplied by: that
// value then lies below 2^12 (as the first operands' does), from 2^11 on where it is below 1, and no value leaves fp16's range.
__host__ __device__ inline int scale_exp(float top) {
  int e;
  frexpf(top, &e);
  return min(15 - e, 12 - min(e, 0));
}

// Step k's factors for one matrix.  Where |G| is not far below eps they are the call's; where it is, X starts small and
// grows by about `a` a step, and its operands are scaled by their own bounds, so that they keep all their bits.  (Factors
// that underflow belong to terms that are nothing beside a X.)
__device__ __noinline__ Factors small_factors(const Steps& p, int k, const Scale& sc) {
  float top = sc.norm;
  for (int i = 0; i < k; ++i) {
    const float q = top * top;
    top = fminf(1.001f * top * fmaf(q, fmaf(q, fabsf(p.c), fabsf(p.b)), fabsf(p.a)), p.step[i + 1].top);
  }
  const float q = top * top, next = 1.001f * top * fmaf(q, fmaf(q, fabsf(p.c), fabsf(p.b)), fabsf(p.a));
  int e;
  const float t = frexpf(1.1f * top, &e);  // (squares may underflow: their exponents are counted apart)
  const int sa = scale_exp(t * t) - 2 * e, sb = scale_exp(1.1f * fmaf(q, fabsf(p.c), fabsf(p.b)) * t * t) - 2 * e;
  const int sx = scale_exp(1.1f * top), sx1 = k + 1 == p.n ? 0 : scale_exp(1.1f * fminf(next, p.step[k + 1].top));
  Factors f;
  f.square_acc = ldexpf(p.c, sb - 2 * sa);
  f.square_old = ldexpf(p.b, sb - sa);
  if (k == 0) {
    const int h = sa / 2;
    const float r = ldexpf(sc.rho, h);
    f.gram = ldexpf(r * r, sa - 2 * h);
    f.apply_acc = ldexpf(sc.rho, sx1 - sb);
    f.apply_old = p.a * ldexpf(sc.rho, sx1);
  } else {
    f.gram = ldexpf(1.f, sa - 2 * sx);
    f.apply_acc = ldexpf(1.f, sx1 - sb - sx);
    f.apply_old = ldexpf(p.a, sx1 - sx);
  }
  return f;
}
__device__ __forceinline__ bool is_small(const Scale& sc) { return sc.norm < 0.5f && sc.norm > 0.f; }
__device__ __forceinline__ Factors factors_of(const Steps& p, int k, const Scale& sc) {
  if (is_small(sc)) return small_factors(p, k, sc);
  Factors f = p.step[k].f;
  if (k == 0) {
    f.gram *= sc.rho * sc.rho;
    f.apply_acc *= sc.rho;
    f.apply_old *= sc.rho;
  }
  return f;
}

// The block's sum of squares, in every thread of its first warp.
__device__ __forceinline__ Squares block_sum(Squares q, Squares* part) {
  q = warp_sum(q);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = q;
  __syncthreads();
  q = Squares{};
  if (threadIdx.x < blockDim.x / 32) q = part[threadIdx.x];
  return threadIdx.x < 32 ? warp_sum(q) : q;
}

struct Input {
  const void* g;
  int64_t sb, sr;
  int rows, cols;
};

// Eight consecutive values, by one or two 16-byte loads where `aligned`.
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool aligned, int n, float (&v)[8]) {
  if (aligned && n >= 8) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const uint4 w = *reinterpret_cast<const uint4*>(p);
      const T* h = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = to_f32(h[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? to_f32(p[j]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ bool rows_aligned(const Input& in) {
  constexpr int kPer = 16 / sizeof(T);
  return ((uintptr_t)in.g & 15) == 0 && in.sr % kPer == 0 && in.sb % kPer == 0;
}

// The sum of squares of block blockIdx.x's share of rows of matrix blockIdx.y, eight values a thread at a time.
template <typename T>
__global__ void __launch_bounds__(256) k_orth_squares(const Input in, Squares* part) {
  __shared__ Squares s_part[8];
  const T* g = (const T*)in.g + blockIdx.y * in.sb;
  const bool aligned = rows_aligned<T>(in);
  const int pieces = (in.cols + 7) / 8, per = pieces < 256 ? 256 / pieces : 1;  // rows side by side
  const int r0 = threadIdx.x / (per > 1 ? pieces : 256), p0 = per > 1 ? threadIdx.x % pieces : threadIdx.x;
  Squares q;
  if (r0 < per)
    for (int64_t r = (int64_t)blockIdx.x * per + r0; r < in.rows; r += (int64_t)gridDim.x * per)
#pragma unroll 2
      for (int c = p0; c < pieces; c += 256) {
        float v[8];
        load8(g + r * in.sr + 8 * c, aligned, in.cols - 8 * c, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) q.add(v[j]);
      }
  const Squares sum = block_sum(q, s_part);
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// A matrix's partial sums -> its scale and, [step][product][matrix], what its products' sums and old values are multiplied
// by.  (One warp a matrix, sums in a fixed order; a step a lane.)
__global__ void __launch_bounds__(32) k_orth_scale(const Squares* part, int nparts, float eps, const __grid_constant__ Steps steps,
                                                   Scale* scale, float2* factors) {
  Squares q;
#pragma unroll 4
  for (int i = threadIdx.x; i < nparts; i += 32) q.add(part[(int64_t)blockIdx.x * nparts + i]);
  q = warp_sum(q);
  const Scale sc = scale_of(q, eps);
  if (threadIdx.x == 0) scale[blockIdx.x] = sc;
  const int k = threadIdx.x;
  if (k < steps.n) {
    const Factors f = factors_of(steps, k, sc);
    float2* const to = factors + (int64_t)k * 3 * gridDim.x + blockIdx.x;
    to[0] = make_float2(f.gram, 0.f);
    to[gridDim.x] = make_float2(f.square_acc, f.square_old);
    to[2 * (int64_t)gridDim.x] = make_float2(f.apply_acc, f.apply_old);
  }
}

// v as one or two fp16 parts.
__device__ __forceinline__ __half hi_part(float v) { return __float2half_rn(v); }
__device__ __forceinline__ __half lo_part(float v, __half hi) { return __float2half_rn(v - __half2float(hi)); }

// A matrix of fp16 parts in scratch memory: [part][matrix of the batch][rows][ld].
struct Parts {
  __half* p;
  int64_t ld, matrix, part;  // elements
  int parts;
};

// Eight consecutive values of a row.  (Rows are padded to whole groups of eight.)
__device__ __forceinline__ void store_parts8(const Parts& to, int64_t at, const float (&v)[8]) {
  __half2 h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
    const float2 f = __half22float2(h[j]);
    l[j] = __floats2half2_rn(v[2 * j] - f.x, v[2 * j + 1] - f.y);
  }
  *reinterpret_cast<uint4*>(to.p + at) = *reinterpret_cast<const uint4*>(h);
  if (to.parts > 1) *reinterpret_cast<uint4*>(to.p + at + to.part) = *reinterpret_cast<const uint4*>(l);
}

// The first operands from G: X and X^T, by 64 x 64 tiles through shared memory (blockIdx.z: matrix).
template <typename T>
__global__ void __launch_bounds__(256) k_orth_first(const Input in, const Scale* scale, bool flip, Parts x, Parts xt) {
  __shared__ float tile[64][65];
  const Scale sc = scale[blockIdx.z];
  const T* g = (const T*)in.g + blockIdx.z * in.sb;
  const bool aligned = rows_aligned<T>(in);
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, piece = (threadIdx.x & 7) * 8;
  const Parts &a = flip ? xt : x, &b = flip ? x : xt;  // G's own orientation, and the other
#pragma unroll
  for (int i = threadIdx.x >> 3; i < 64; i += 32) {
    const int r = r0 + i, c = c0 + piece;
    float v[8] = {};
    if (r < in.rows && c < in.cols) {
      load8(g + r * in.sr + c, aligned, in.cols - c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] * sc.s0 * sc.s1;
      store_parts8(a, blockIdx.z * a.matrix + r * a.ld + c, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[i][piece + j] = v[j];
  }
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.x >> 3; i < 64; i += 32) {
    const int r = c0 + i, c = r0 + piece;
    if (r < in.cols && c < in.rows) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = tile[piece + j][i];
      store_parts8(b, blockIdx.z * b.matrix + r * b.ld + c, v);
    }
  }
}

// steps = 0: G / (|G|_F + eps).
template <typename T>
__global__ void __launch_bounds__(256) k_orth_scaled(const Input in, const Scale* scale, T* out, int64_t sb, int64_t sr) {
  const Scale sc = scale[blockIdx.y];
  for (int r = blockIdx.x; r < in.rows; r += gridDim.x)
    for (int c = threadIdx.x; c < in.cols; c += blockDim.x)
      out[blockIdx.y * sb + r * sr + c] = from_f32<T>(to_f32(((const T*)in.g)[blockIdx.y * in.sb + r * in.sr + c]) * sc.s0 * sc.s1 * sc.rho);
}

// ------------------------------------------------------------------------------------------
// The products on the tensor cores
// ------------------------------------------------------------------------------------------

// K-major operand tiles of rows of BK fp16 values (128 or 64 bytes), swizzled as the tensor copies write them:
// groups of 8 rows follow each other.
template <int BK>
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr) {
  constexpr uint64_t group = 8 * BK * 2, layout = BK == 64 ? 2 : 4;  // 128- or 64-byte swizzle
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (1ull << 16) | ((group >> 4) << 32) | (1ull << 46) | (layout << 61);
}
// kind::f16: fp16 A and B, fp32 D.
__host__ __device__ constexpr uint32_t product_idesc(int n, int m = 128) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// CTAS = 2: the pair's first block issues for both, on operands at the same offsets of their shared memories.
template <int CTAS = 1>
__device__ __forceinline__ void product_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if constexpr (CTAS == 1)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a),
        "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a),
        "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// Completion of the products issued so far, to the barrier (CTAS = 2: to that of both blocks).
template <int CTAS = 1>
__device__ __forceinline__ void product_commit(uint64_t* bar) {
  if constexpr (CTAS == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_u32(bar)) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(shared_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t* to, uint32_t columns) {
  if constexpr (CTAS == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_u32(to)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_u32(to)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
  if constexpr (CTAS == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
// A tensor copy of one of a pair's blocks that reports to a barrier of either (cluster address).
__device__ __forceinline__ void tma_load_pair(void* to, const CUtensorMap* map, int32_t c0, int32_t c1, int32_t c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          shared_u32(to)),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void accum_load(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
               "tcgen05.wait::ld.sync.aligned;"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void accum_ask16(uint32_t taddr, uint32_t (&r)[16]) {  // (until accum_wait)
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr) : "memory");
}
// The registers are tied to the wait, so no use of them is scheduled before it.
__device__ __forceinline__ void accum_wait16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :: "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void barrier_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_u32(bar)) : "memory");
}
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}

constexpr int kTileM = 128;
// A copying warp, an issuing warp, and epilogue warps: four where a pair's products take longer than the blocks of the
// tile before, which another accumulator holds; eight where a tile's blocks are waited for.
__host__ __device__ constexpr int epilogue_warps(int ctas, int bk) { return ctas == 2 && bk == 64 ? 4 : 8; }
__host__ __device__ constexpr int mma_threads(int ctas, int bk) { return 64 + 32 * epilogue_warps(ctas, bk); }
// The tensor cores truncate where they add to an accumulator (about 2^-24 of it each time, always towards zero).  So the
// sums of results that are held to fp32 leave tensor memory every few stages (three additions per 16 of depth) and are
// added up in the epilogue warps' registers, rounded to nearest.  In one accumulator 4096 x 1024 came out 1.1e-5 off (fp32
// arithmetic: 6e-6); with the cross products in one of their own 4096 x 4096 still 3e-5 (1.2e-5); every 256 of depth 2e-6,
// for a tenth more time.  Short sums, whose size the rest of the error does not hide, leave every 128.  bf16 results need
// it only for sums so long (kLongSum) that the truncations reach their rounding; there operands of one part take the
// same way, and so do those of fp16 results, whose first step is exact but for this (3 x 200000: 4.2e-4 off, with it 2.1e-4; at
// kLongSum 1024 truncations of half 2^-24 leave 3e-5 beside the rounding's 2.1e-4).
constexpr int kNoChunks = 1 << 30, kLongSum = 16384;
inline int chunk_of(int type, int depth) {
  return type != MF_TYPE_BF16 ? (depth <= 1024 ? 4 : 8) : depth <= kLongSum ? kNoChunks : 64;
}

enum Epilogue { kGram, kSquare, kApply, kFinal };

// The bounded waits of a call.  mf_debug_operators_wait_test: a wait runs out at the start, after `polls` tests, and later ones
// expect bytes or arrivals that nothing sends; else both are 0.
struct Waits {
  uint32_t polls, unsent;
  uint32_t* status;
};

struct Product {
  int rows, cols, depth;        // of the result, and of the sum
  int batch, na, nb;            // matrices; parts of the operands
  int tiles_r, tiles_c, tiles;  // tiles of a matrix (rows, columns), those that are computed of the whole batch
  int chunk;                    // stages of a sum's part (split operands)
  int splits;                   // blocks of a cluster that share a tile's depth (1: none)
  bool symmetric;
  const float2* factors;        // of each matrix: result = x * sum + y * old
  Parts old, out, out_t;        // out_t: the transposed result (kApply), or out itself (symmetric)
  void* final_out;
  int64_t final_sb, final_sr;
  bool flip;                    // kFinal: the result is written transposed
  Waits waits;
};

// Wait on a barrier; false (for good: *gave_up) once a wait of the block has run out, after 4096 tests of a millisecond
// at most.  (With the limit as an argument, or in shared memory, the products of pairs took 2 % longer.)
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile int* gave_up, uint32_t* status) {
  for (uint32_t tries = 0; !barrier_test(bar, parity); ++tries) {
    if (*gave_up) return false;
    if (tries >= 4096) {
      *gave_up = 1;
      if (status) atomicOr(status, kStatusTimeout);
      return false;
    }
  }
  return true;
}
// A wait of `polls` tests that runs out (nothing has arrived at the barrier).
__device__ __noinline__ void run_out(uint64_t* bar, uint32_t polls, volatile int* gave_up, uint32_t* status) {
  for (uint32_t n = 0; n < polls && !barrier_test(bar, 0); ++n) {}
  *gave_up = 1;
  if (status) atomicOr(status, kStatusTimeout);
}

// Tile `t` of the batch -> (matrix, first row, first column).  Symmetric results: only tiles that reach the diagonal, row
// by row of tiles.
template <int TM, int BN>
__device__ __forceinline__ void tile_of(const Product& p, int t, int& matrix, int& r0, int& c0) {
  const int per = p.tiles / p.batch;
  matrix = t / per;
  int i = t - matrix * per;
  if (!p.symmetric) {
    r0 = i % p.tiles_r * TM;  // (down a column of tiles: neighbours share the wider operand)
    c0 = i / p.tiles_r * BN;
    return;
  }
  int r = 0;
  for (;; ++r) {
    const int n = min(p.tiles_c, (r * TM + TM - 1) / BN + 1);
    if (i < n) break;
    i -= n;
  }
  r0 = r * TM;
  c0 = i * BN;
}

// An epilogue warp's shared memory: 32 x 32 blocks of fp16 parts, rows of 64 bytes.
struct WarpBlocks {
  uint4 out[2][128];     // [part], 64-byte swizzle; kFinal: the block in fp32
  uint4 old[2][128];     // [part], 64-byte swizzle
  __half out_t[2][1024]; // [part], transposed
};
__host__ __device__ constexpr uint32_t blocks_bytes(int epi) {
  return epi == kGram || epi == kFinal ? 8192 : sizeof(WarpBlocks);  // (kGram has no old, kFinal no out_t)
}
// A stage: 128 rows of A, BN / CTAS of B, 64 values deep, or 32 of two parts each; as many as fit.
constexpr uint32_t kMostShared = 227 * 1024 - 1024;  // (static variables beside)
__host__ __device__ constexpr uint32_t stage_bytes(int ctas, int bn) { return (uint32_t)(kTileM + bn / ctas) * 128; }
__host__ __device__ constexpr int stages_of(int ctas, int bn, int bk, int epi) {
  return (int)((kMostShared - 1024 - epilogue_warps(ctas, bk) * blocks_bytes(epi)) / stage_bytes(ctas, bn));
}
__host__ __device__ constexpr uint32_t shared_of(int ctas, int bn, int bk, int epi) {
  return stages_of(ctas, bn, bk, epi) * stage_bytes(ctas, bn) + epilogue_warps(ctas, bk) * blocks_bytes(epi) + 1024;
}

// 16-byte piece `g` of row `row` of a block of 64-byte rows as 64-byte-swizzled tensor copies lay it out.
__device__ __forceinline__ int piece(int row, int g) { return row * 4 + (g ^ ((row >> 1) & 3)); }

__device__ __forceinline__ void add_halves(const uint4& w, float (&v)[8]) {
  const __half2* h = reinterpret_cast<const __half2*>(&w);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = __half22float2(h[j]);
    v[2 * j] += f.x;
    v[2 * j + 1] += f.y;
  }
}

struct MmaMaps {
  CUtensorMap a, b, old, out, out_t;
};

// A warp's 32 rows of a tile's accumulator from block column c (matrix coordinates row0, col0): acc -> the result.
template <int EPI, typename T>
__device__ __forceinline__ void finish_block(const Product& p, const MmaMaps& maps, WarpBlocks& w, __half (*out_t)[1024], int matrix, int row0,
                                             int col0, const uint32_t (&acc)[32], float f_acc, float f_old) {
  const int lane = threadIdx.x & 31;
  if constexpr (EPI != kFinal) {
    // the stores of the block before have read their buffers
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  }
  __syncwarp();
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float v[8];
    if constexpr (EPI == kGram) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = f_acc * __uint_as_float(acc[8 * g + j]);
    } else {
      float old[8] = {};
      add_halves(w.old[0][piece(lane, g)], old);
      if (p.old.parts > 1) add_halves(w.old[1][piece(lane, g)], old);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = fmaf(f_acc, __uint_as_float(acc[8 * g + j]), f_old * old[j]);
    }
    if constexpr (EPI == kFinal) {
      T* out = (T*)p.final_out + matrix * p.final_sb;
      if (p.flip) {  // lanes lie along the rows of the result
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col0 + 8 * g + j < p.cols && row0 + lane < p.rows) out[(col0 + 8 * g + j) * p.final_sr + row0 + lane] = from_f32<T>(v[j]);
      } else {
        float* f = reinterpret_cast<float*>(w.out);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[lane * 32 + ((8 * g + j) ^ lane)] = v[j];
      }
    } else {
      __half2 h[4], l[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[j] = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
        const float2 f = __half22float2(h[j]);
        l[j] = __floats2half2_rn(v[2 * j] - f.x, v[2 * j + 1] - f.y);
      }
      w.out[0][piece(lane, g)] = *reinterpret_cast<const uint4*>(h);
#pragma unroll
      for (int j = 0; j < 8; ++j) out_t[0][(8 * g + j) * 32 + lane] = j & 1 ? __high2half(h[j / 2]) : __low2half(h[j / 2]);
      if (p.out.parts > 1) {
        w.out[1][piece(lane, g)] = *reinterpret_cast<const uint4*>(l);
#pragma unroll
        for (int j = 0; j < 8; ++j) out_t[1][(8 * g + j) * 32 + lane] = j & 1 ? __high2half(l[j / 2]) : __low2half(l[j / 2]);
      }
    }
  }
  if constexpr (EPI == kFinal) {
    __syncwarp();
    if (!p.flip) {
      T* out = (T*)p.final_out + matrix * p.final_sb;
      const float* f = reinterpret_cast<const float*>(w.out);
      if (col0 + lane < p.cols)
        for (int r = 0; r < 32 && row0 + r < p.rows; ++r) out[(row0 + r) * p.final_sr + col0 + lane] = from_f32<T>(f[r * 32 + (lane ^ r)]);
    }
    __syncwarp();
  } else {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      // (symmetric: a block on the diagonal is its own mirror)
      for (int q = 0; q < p.out.parts; ++q) {
        tma_store_3d(&maps.out, col0, row0, q * p.batch + matrix, w.out[q]);
        if (EPI == kApply || col0 != row0) tma_store_3d(&maps.out_t, row0, col0, q * p.batch + matrix, out_t[q]);
      }
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
}

// D = P Q^T by tiles of 128 CTAS x BN.  A block walks its tiles: a warp copies operand tiles to a ring of stages, a lane
// of another issues the products into one of two accumulators in tensor memory, the epilogue warps finish the other one.
// CTAS = 2: a pair of blocks (two SMs) works on a tile of 256 x 256: each holds its 128 rows of both operands and of the
// result, so an SM reads and copies half as much shared memory a product, which is what bounds tiles of one SM.
// splits > 1 (CTAS = 1): that many blocks of a cluster share a tile's depth; each leaves its sums in its shared
// memory, and each finishes its share of the tile's blocks from all of them, in the order of their ranks.
// Measured: 4096 x 4096, five steps, bf16 1.86 ms by itself (1.48 PFLOP/s of issued products, 0.78 of the measured bf16 burst
// rate) and 2.0 ms in a loop, under the power cap, fp32 2.90 ms (1.42 PFLOP/s), fp16 2.78 ms; of the rest, rounds of 256 x
// 256 tiles that do not fill the last one take a tenth.  Small products are a chain of latencies: 7.5 us each at 256 x 256
// (start 1.5, products 1.8, blocks 1.3, end and the next launch 2 to 3).
template <int CTAS, int BN, int BK, int EPI, typename T>
__global__ void __launch_bounds__(mma_threads(CTAS, BK), 1) k_orth_mma(const Product p, const __grid_constant__ MmaMaps maps) {
  extern __shared__ uint8_t s_raw[];
  uint8_t* const ring = s_raw + ((1024 - (shared_u32(s_raw) & 1023)) & 1023);
  constexpr int kStages = stages_of(CTAS, BN, BK, EPI), kWarps = epilogue_warps(CTAS, BK), kSides = kWarps / 4;
  constexpr uint32_t kStageBytes = stage_bytes(CTAS, BN);
  __shared__ uint64_t s_full[kStages], s_free[kStages], s_done[2], s_taken[2], s_old[kWarps];
  __shared__ uint32_t s_tmem;
  __shared__ int s_gave_up;
  constexpr int kRowsB = BN / CTAS;
  constexpr uint32_t a_bytes = kTileM * BK * 2, b_bytes = kRowsB * BK * 2;
  static_assert((BK == 64 ? 1 : 2) * (a_bytes + b_bytes) == kStageBytes, "a stage holds both operands");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cluster = CTAS == 2 ? 2 : p.splits, rank = cluster > 1 ? (int)cluster_rank() : 0;
  const int first = (int)blockIdx.x / cluster, step = (int)gridDim.x / cluster;

  if (threadIdx.x == 0) {
    s_gave_up = 0;
    for (int i = 0; i < kStages; ++i) {
      barrier_init(&s_full[i], 1);
      barrier_init(&s_free[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(&s_done[i], 1);
      barrier_init(&s_taken[i], 32 * kWarps * CTAS);
    }
    for (int w = 0; w < kWarps; ++w) barrier_init(&s_old[w], 1);
    barrier_init_fence();
    if (p.waits.polls) run_out(&s_done[0], p.waits.polls, &s_gave_up, p.waits.status);
  }
  if (threadIdx.x == 32) {
    for (const CUtensorMap* m : {&maps.a, &maps.b, &maps.old, &maps.out, &maps.out_t})
      asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<CTAS>(&s_tmem, 2 * BN);
  fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync();
  fence_after();
  const uint32_t tmem = s_tmem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");  // what the launch before wrote is there, and it reads nothing more

  const int depth = (p.depth + BK - 1) / BK;  // in stages; this block's are [k0, k1)
  const int k0 = CTAS == 2 ? 0 : depth * rank / p.splits, k1 = CTAS == 2 ? depth : depth * (rank + 1) / p.splits;
  if (warp == 0) {
    if (elected()) {
      asm volatile("fence.proxy.async;" ::: "memory");  // (the operands were written by ordinary stores)
      uint32_t it = 0;
      for (int t = first; t < p.tiles; t += step) {
        int matrix, r0, c0;
        tile_of<kTileM * CTAS, BN>(p, t, matrix, r0, c0);
        if (CTAS == 2) {
          r0 += rank * kTileM;
          c0 += rank * kRowsB;
        }
        for (int k = k0; k < k1; ++k, ++it) {
          const int s = it % kStages;
          if (it >= kStages && !wait_for(&s_free[s], (it / kStages - 1) & 1, &s_gave_up, p.waits.status)) goto copied;
          uint8_t* to = ring + s * kStageBytes;
          if (rank == 0 || CTAS == 1) barrier_expect(&s_full[s], CTAS * (p.na * a_bytes + p.nb * b_bytes) + (EPI == kGram ? p.waits.unsent : 0));
          if constexpr (CTAS == 1) {
            for (int q = 0; q < p.na; ++q) tma_load_3d(to + q * a_bytes, &maps.a, k * BK, r0, q * p.batch + matrix, &s_full[s]);
            for (int q = 0; q < p.nb; ++q)
              tma_load_3d(to + p.na * a_bytes + q * b_bytes, &maps.b, k * BK, c0, q * p.batch + matrix, &s_full[s]);
          } else {
            const uint32_t bar = in_block(&s_full[s], 0);
            for (int q = 0; q < p.na; ++q) tma_load_pair(to + q * a_bytes, &maps.a, k * BK, r0, q * p.batch + matrix, bar);
            for (int q = 0; q < p.nb; ++q)
              tma_load_pair(to + p.na * a_bytes + q * b_bytes, &maps.b, k * BK, c0, q * p.batch + matrix, bar);
          }
        }
      }
    copied:;
    }
    __syncwarp();
  } else if (warp == 1) {
    if ((CTAS == 1 || rank == 0) && elected()) {
      constexpr uint32_t idesc = product_idesc(BN, kTileM * CTAS);
      uint32_t it = 0, n = 0;
      for (int t = first; t < p.tiles; t += step) {
        for (int k = k0; k < k1; ++n) {
          const uint32_t u = n & 1, d = tmem + u * BN;
          if (n >= 2 && !wait_for(&s_taken[u], (n / 2 - 1) & 1, &s_gave_up, p.waits.status)) goto issued;
          fence_after();
          const int begin = k, end = BK == 32 && k1 - k > p.chunk ? k + p.chunk : k1;
          for (; k < end; ++k, ++it) {
            const int s = it % kStages;
            if (!wait_for(&s_full[s], (it / kStages) & 1, &s_gave_up, p.waits.status)) goto issued;
            fence_after();
            const uint32_t a = shared_u32(ring + s * kStageBytes), b = a + p.na * a_bytes;
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
              const uint64_t da = operand_desc<BK>(a + kk * 32), db = operand_desc<BK>(b + kk * 32);
              product_mma<CTAS>(d, da, db, idesc, k > begin || kk > 0);
              if constexpr (BK == 32) {
                if (p.nb > 1) product_mma<CTAS>(d, da, operand_desc<BK>(b + b_bytes + kk * 32), idesc, true);
                if (p.na > 1) product_mma<CTAS>(d, operand_desc<BK>(a + a_bytes + kk * 32), db, idesc, true);
              }
            }
            product_commit<CTAS>(&s_free[s]);
          }
          product_commit<CTAS>(&s_done[u]);
        }
      }
    issued:;
    }
    __syncwarp();
  }
  // (a warp reaches the 32 tensor-memory lanes of its number mod 4; two of them share a tile's blocks by turns)
  const int quarter = warp & 3, own = warp >= 2 ? warp - 2 : 0, side = own >> 2;
  WarpBlocks& w = *reinterpret_cast<WarpBlocks*>(ring + kStages * kStageBytes + own * blocks_bytes(EPI));
  __half(*const out_t)[1024] = EPI == kGram ? reinterpret_cast<__half(*)[1024]>(w.old) : w.out_t;
  // blocks of `old`; the top bit once a wait for one has given up: its phase may not have ended, and takes no second arrival
  uint32_t uses = 0;
  if (warp >= 2) {
    uint32_t n = 0;
    const auto taken = [&](uint32_t u) {  // (this thread has read accumulator u)
      fence_before();
      if (CTAS == 2 && rank == 1)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_block(&s_taken[u], 0)) : "memory");
      else
        barrier_arrive(&s_taken[u]);
    };
    for (int t = first; t < p.tiles; t += step) {
      int matrix, r0, c0;
      tile_of<kTileM * CTAS, BN>(p, t, matrix, r0, c0);
      const int row0 = r0 + (CTAS == 2 ? rank * kTileM : 0) + quarter * 32;
      // this quarter's blocks: those with a column of the matrix, symmetric: up to the diagonal
      int blocks = row0 >= p.rows ? 0 : (min(BN, p.cols - c0) + 31) / 32;
      if (p.symmetric) blocks = max(0, min(blocks, (row0 - c0) / 32 + 1));
      const bool shared = CTAS == 1 && p.splits > 1;  // by a cluster's blocks, whose sums meet first
      const int b0 = shared ? rank + p.splits * side : side, every = shared ? p.splits * kSides : kSides;
      const auto load_old = [&](int i) {
        if (EPI == kGram || lane != 0 || i >= blocks || (int)uses < 0) return;
        barrier_expect(&s_old[own], (uint32_t)p.old.parts * 2048 + p.waits.unsent);
        for (int q = 0; q < p.old.parts; ++q)
          tma_load_3d(w.old[q], &maps.old, c0 + 32 * i, row0, q * p.batch + matrix, &s_old[own]);
      };
      load_old(b0);
      const float2 factors = p.factors[matrix];
      const auto finish = [&](int i, const uint32_t (&acc)[32]) {
        if (EPI != kGram && !wait_for(&s_old[own], uses & 1, &s_gave_up, p.waits.status)) uses |= 1u << 31;
        ++uses;
        finish_block<EPI, T>(p, maps, w, out_t, matrix, row0, c0 + 32 * i, acc, factors.x, factors.y);
        __syncwarp();
        load_old(i + every);
      };
      const uint32_t sums_at = tmem + ((uint32_t)quarter << 21);
      if constexpr (BK == 64) {
        const uint32_t u = n & 1;
        const bool there = wait_for(&s_done[u], (n / 2) & 1, &s_gave_up, p.waits.status);
        ++n;
        fence_after();
        if (!shared) {
          if (!there) break;
          for (int i = b0; i < blocks; i += every) {
            uint32_t acc[32];
            __syncwarp();
            accum_load(sums_at + u * BN + 32 * i, acc);
            finish(i, acc);
          }
        } else {
          float* sums = reinterpret_cast<float*>(ring) + quarter * 1024 + lane;  // [block][quarter][column][row]
          for (int i = side; i < blocks; i += kSides) {
            uint32_t acc[32];
            __syncwarp();
            accum_load(sums_at + u * BN + 32 * i, acc);
#pragma unroll
            for (int j = 0; j < 32; ++j) sums[i * 4096 + j * 32] = __uint_as_float(acc[j]);
          }
        }
        taken(u);
      } else {
        constexpr int kOwn = BN / 32 / kSides;  // blocks of a warp, in registers
        uint32_t sum[kOwn][32];
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
#pragma unroll
          for (int e = 0; e < 32; ++e) sum[j][e] = 0u;
        bool there = true;
        for (int k = k0; k < k1; k = k1 - k > p.chunk ? k + p.chunk : k1, ++n) {
          const uint32_t u = n & 1;
          there = there && wait_for(&s_done[u], (n / 2) & 1, &s_gave_up, p.waits.status);
          fence_after();
#pragma unroll
          for (int j = 0; j < kOwn; ++j) {
            if (side + kSides * j < blocks) {
              uint32_t acc[32];
              __syncwarp();
              accum_load(sums_at + u * BN + 32 * (side + kSides * j), acc);
#pragma unroll
              for (int e = 0; e < 32; ++e) sum[j][e] = __float_as_uint(__uint_as_float(sum[j][e]) + __uint_as_float(acc[e]));
            }
          }
          taken(u);
        }
        if (!shared) {
          if (!there) break;
#pragma unroll
          for (int j = 0; j < kOwn; ++j)
            if (side + kSides * j < blocks) finish(side + kSides * j, sum[j]);
        } else {
          float* sums = reinterpret_cast<float*>(ring) + quarter * 1024 + lane;
#pragma unroll
          for (int j = 0; j < kOwn; ++j)
            if (side + kSides * j < blocks)
#pragma unroll
              for (int e = 0; e < 32; ++e) sums[(side + kSides * j) * 4096 + e * 32] = __uint_as_float(sum[j][e]);
        }
      }
      if (shared) {  // (one tile a block: every copy and product of this block is done, so the ring was free)
        asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
        const float* sums = reinterpret_cast<const float*>(ring) + quarter * 1024 + lane;
        for (int i = b0; i < blocks; i += every) {
          uint32_t acc[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) acc[j] = 0u;
          for (int r = 0; r < p.splits; ++r) {
            const uint32_t from = in_block(sums + i * 4096, (uint32_t)r);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              float v;
              asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(from + j * 128));
              acc[j] = __float_as_uint(__uint_as_float(acc[j]) + v);
            }
          }
          finish(i, acc);
        }
      }
    }
    // (the buffers have to outlast the stores' reads; what they write is there when the grid has ended)
    if (EPI != kFinal && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  } else if (CTAS == 1 && p.splits > 1) {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
  }
  __syncthreads();
  if (s_gave_up) {  // copies and products in flight end before the memory that they use is given back
    const unsigned long long until = device_ns() + 20000000ull;
    while (device_ns() < until) {}
  }
  __syncthreads();
  if (cluster > 1) cluster_sync();  // (nobody reads another block's shared memory or works on its tensor memory any more)
  if (warp == 1) tmem_free<CTAS>(tmem, 2 * BN);
}

// ------------------------------------------------------------------------------------------
// Small matrices: all steps of one in one block
// ------------------------------------------------------------------------------------------

// X, X^T and A (whose room B takes over) stay in shared memory as operands, each in panels of 64 values of depth (rows of
// 128 bytes, 128-byte swizzle); sums go to tensor memory and come back a row a thread, which reads its old values and writes
// the new ones in place.  What bounds it is the chain of 3 `steps` products, each a rendezvous, a product (75 cycles an
// instruction of 16 deep), a read-back and a write: in fp32 1.4 us at 64 x 64 (5 matrices 27 us), 3.4 us at 128 x 128 (one 56 us).
// Rows up to the next multiple of 16 are kept as zeros; tensor memory's lanes above them hold sums of whatever lies behind an
// operand's rows and are never read.
struct Small {
  Input in;
  void* out;
  int64_t out_sb, out_sr;
  int64_t batch;
  int m, n, mp, np, first_parts;
  bool flip;
  float eps;
  uint32_t xoff, toff;    // of X and X^T after A, bytes
  uint32_t ap, xp, tp;    // bytes of a part of each
  uint32_t columns;       // of tensor memory
  uint32_t cross;         // columns from a sum to that of its cross products (0: one sum, where there is no room for two)
  Waits waits;
  Steps steps;
};

// Offset of value k of row r in an operand of `rows` rows.
__device__ __forceinline__ uint32_t small_at(int r, int k, int rows) {
  return ((uint32_t)(k >> 6) * rows + r) * 128 + ((((k >> 3) & 7) ^ (r & 7)) << 4) + (k & 7) * 2;
}

constexpr int kSmallThreads = 512;

// One product of 128 x cols with depth `depth` (multiples of 16) of operands at a and b (shared addresses; rows of each).
__device__ __forceinline__ void small_product(uint32_t d, uint32_t a, uint32_t a_part, int a_rows, int na, uint32_t b, uint32_t b_part,
                                              int b_rows, int nb, int cols, int depth, uint32_t cross, uint64_t* done) {
  const uint64_t la = a_part >> 4, lb = b_part >> 4;  // (descriptors count 16 bytes)
  for (int c = 0; c < cols; c += 256) {
    const uint32_t idesc = product_idesc(min(256, cols - c));
    uint64_t da = operand_desc<64>(a), db = operand_desc<64>(b + c * 128);
    bool add = false;
    for (int k = depth / 16; k > 0; k -= 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= k) break;
        product_mma(d + c, da + 2 * i, db + 2 * i, idesc, add);
        if (nb > 1) product_mma(d + c + cross, da + 2 * i, db + lb + 2 * i, idesc, add || !cross);
        if (na > 1) product_mma(d + c + cross, da + la + 2 * i, db + 2 * i, idesc, add || nb > 1 || !cross);
        add = true;
      }
      da += a_rows * 8;  // the next panel
      db += b_rows * 8;
    }
  }
  product_commit(done);
}

// A warp's share of a product's sums -> its result (WHAT, and whether it is the call's).
template <int WHAT, bool LAST, typename T>
__device__ __forceinline__ void small_finish(const Small& p, uint8_t* A, uint8_t* X, uint8_t* XT, uint32_t tmem, uint32_t cross,
                                             int64_t matrix, float f_acc, float f_old, int parts, int old_parts) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, row = quarter * 32 + lane;
  if (quarter * 32 >= p.mp) return;
  uint8_t* const to = WHAT == kApply ? X : A;
  const uint32_t part = WHAT == kApply ? p.xp : p.ap;
  const int cols = WHAT == kApply ? p.np : p.mp;
  // of X^T: this row's depth, in rows that start at a multiple of eight
  const uint32_t tcol = (uint32_t)(row >> 6) * p.np * 128 + (row & 7) * 2, tpiece = ((row >> 3) & 7) << 4;
  for (int c0 = (warp >> 2) * 16; c0 < cols; c0 += kSmallThreads / 128 * 16) {
    uint32_t acc[16];
    __syncwarp();
    const uint32_t at_sum = tmem + c0 + ((uint32_t)quarter << 21);
    accum_ask16(at_sum, acc);
    if (cross) {  // (kept out of the large sum, whose additions truncate)
      uint32_t more[16];
      accum_ask16(at_sum + cross, more);
      accum_wait16(more);
      accum_wait16(acc);
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[j] = __float_as_uint(__uint_as_float(acc[j]) + __uint_as_float(more[j]));
    } else {
      accum_wait16(acc);
    }
    if (row >= p.mp) continue;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int c = c0 + 8 * q;
      const uint32_t at = small_at(row, c, p.mp);
      float v[8], old[8] = {};
      if (WHAT != kGram) {
        add_halves(*reinterpret_cast<const uint4*>(to + at), old);
        if (old_parts > 1) add_halves(*reinterpret_cast<const uint4*>(to + part + at), old);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = fmaf(f_acc, __uint_as_float(acc[8 * q + j]), f_old * old[j]);
      if constexpr (LAST) {
        if (p.flip) {  // lanes lie along the result's rows
          T* out = (T*)p.out + matrix * p.out_sb;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (row < p.m && c + j < p.n) out[(c + j) * p.out_sr + row] = from_f32<T>(v[j]);
        } else {  // in fp32 where both parts of the eight values were
          *reinterpret_cast<float4*>(X + at) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4*>(X + p.xp + at) = make_float4(v[4], v[5], v[6], v[7]);
        }
      } else {
      __half2 h[4], l[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[j] = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
        const float2 f = __half22float2(h[j]);
        l[j] = __floats2half2_rn(v[2 * j] - f.x, v[2 * j + 1] - f.y);
      }
      *reinterpret_cast<uint4*>(to + at) = *reinterpret_cast<const uint4*>(h);
      if (parts > 1) *reinterpret_cast<uint4*>(to + part + at) = *reinterpret_cast<const uint4*>(l);
      if constexpr (WHAT == kApply) {
        uint8_t* const t = XT + tcol + c * 128;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint8_t* const e = t + j * 128 + (tpiece ^ (j << 4));
          *reinterpret_cast<__half*>(e) = j & 1 ? __high2half(h[j / 2]) : __low2half(h[j / 2]);
          if (parts > 1) *reinterpret_cast<__half*>(e + p.tp) = j & 1 ? __high2half(l[j / 2]) : __low2half(l[j / 2]);
        }
      }
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kSmallThreads, 2) k_orth_small(const __grid_constant__ Small p) {
  extern __shared__ uint8_t s_raw[];
  uint8_t* const base = s_raw + ((1024 - (shared_u32(s_raw) & 1023)) & 1023);
  __shared__ Squares s_part[kSmallThreads / 32];
  __shared__ Scale s_scale;
  __shared__ Factors s_factors[MF_ORTH_MAX_STEPS];
  __shared__ uint64_t s_done;
  __shared__ uint32_t s_tmem;
  __shared__ int s_gave_up;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    s_gave_up = 0;
    barrier_init(&s_done, 1 + p.waits.unsent);
    barrier_init_fence();
    if (p.waits.polls) run_out(&s_done, p.waits.polls, &s_gave_up, p.waits.status);
  }
  if (warp == 0) {
    tmem_alloc<1>(&s_tmem, p.columns);
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  uint8_t *const A = base, *const X = base + p.xoff, *const XT = base + p.toff;
  const uint32_t a_at = shared_u32(A), x_at = shared_u32(X), t_at = shared_u32(XT);
  uint32_t phase = 0;

  for (int64_t matrix = blockIdx.x; matrix < p.batch; matrix += gridDim.x) {
    const T* g = (const T*)p.in.g + matrix * p.in.sb;
    // G by pieces of eight values of a row
    const bool aligned = rows_aligned<T>(p.in);
    const int pieces = (p.in.cols + 7) / 8, all = p.in.rows * pieces;
    Squares sq;
#pragma unroll 4
    for (int i = tid; i < all; i += kSmallThreads) {
      const int r = i / pieces, c = (i - r * pieces) * 8;
      float v[8];
      load8(g + r * p.in.sr + c, aligned, p.in.cols - c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sq.add(v[j]);
    }
    const Squares sum = block_sum(sq, s_part);
    if (tid == 0) s_scale = scale_of(sum, p.eps);
    __syncthreads();
    const Scale sc = s_scale;
    // the first operands, zeros around them: G's own orientation by whole pieces, the other by values (lanes lie along
    // G's columns, so that these go to consecutive places)
    const int rows = p.flip ? p.np : p.mp, cols = p.flip ? p.mp : p.np, around = cols / 8;
    uint8_t *const own = p.flip ? XT : X, *const other = p.flip ? X : XT;
    const uint32_t own_part = p.flip ? p.tp : p.xp, other_part = p.flip ? p.xp : p.tp;
#pragma unroll 2
    for (int i = tid; i < rows * around; i += kSmallThreads) {
      const int r = i % rows, c = i / rows * 8;
      float v[8] = {};
      if (r < p.in.rows && c < p.in.cols) load8(g + r * p.in.sr + c, aligned, p.in.cols - c, v);
      __half h[8], l[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = v[j] * sc.s0 * sc.s1;
        h[j] = hi_part(v[j]);
        l[j] = lo_part(v[j], h[j]);
      }
      const uint32_t at = small_at(r, c, rows);
      *reinterpret_cast<uint4*>(own + at) = *reinterpret_cast<const uint4*>(h);
      if (p.first_parts > 1) *reinterpret_cast<uint4*>(own + own_part + at) = *reinterpret_cast<const uint4*>(l);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t tat = small_at(c + j, r, cols);
        *reinterpret_cast<__half*>(other + tat) = h[j];
        if (p.first_parts > 1) *reinterpret_cast<__half*>(other + other_part + tat) = l[j];
      }
    }
    int xparts = p.first_parts;
    if (tid < p.steps.n) s_factors[tid] = factors_of(p.steps, tid, sc);
    for (int k = 0; k < p.steps.n; ++k) {
      const Step& st = p.steps.step[k];
#pragma unroll 1
      for (int what = kGram; what <= kApply; ++what) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        __syncthreads();
        fence_after();
        if (warp == 0 && elected()) {
          if (what == kGram) small_product(tmem, x_at, p.xp, p.mp, xparts, x_at, p.xp, p.mp, xparts, p.mp, p.np, p.cross, &s_done);
          else if (what == kSquare) small_product(tmem, a_at, p.ap, p.mp, st.parts, a_at, p.ap, p.mp, st.parts, p.mp, p.mp, p.cross, &s_done);
          else small_product(tmem, a_at, p.ap, p.mp, st.parts, t_at, p.tp, p.np, xparts, p.np, p.mp, p.cross, &s_done);
        }
        __syncwarp();
        if (!barrier_polls(&s_done, phase & 1) && !*(volatile int*)&s_gave_up) wait_for(&s_done, phase & 1, &s_gave_up, p.waits.status);
        ++phase;
        fence_after();
        const Factors& f = s_factors[k];
        const float f_acc = what == kGram ? f.gram : what == kSquare ? f.square_acc : f.apply_acc;
        const float f_old = what == kSquare ? f.square_old : f.apply_old;
        // (parts of the product's operands)
        const int na = what == kGram ? xparts : st.parts, nb = what == kSquare ? st.parts : xparts;
        const uint32_t cross = na + nb > 2 ? p.cross : 0;
        if (what == kGram) small_finish<kGram, false, T>(p, A, X, XT, tmem, cross, matrix, f_acc, f_old, st.parts, 0);
        else if (what == kSquare) small_finish<kSquare, false, T>(p, A, X, XT, tmem, cross, matrix, f_acc, f_old, st.parts, st.parts);
        else if (k + 1 < p.steps.n) small_finish<kApply, false, T>(p, A, X, XT, tmem, cross, matrix, f_acc, f_old, st.next_parts, xparts);
        else small_finish<kApply, true, T>(p, A, X, XT, tmem, cross, matrix, f_acc, f_old, 0, xparts);
      }
      xparts = st.next_parts;
    }
    fence_before();
    __syncthreads();  // (every read of the sums is done before the next matrix's products)
    fence_after();
    if (!p.flip) {  // the result, a row a warp
      for (int r = warp; r < p.m; r += kSmallThreads / 32)
        for (int c = lane; c < p.n; c += 32) {
          const float* f = reinterpret_cast<const float*>(X + ((c & 4) ? p.xp : 0) + small_at(r, c & ~7, p.mp));
          ((T*)p.out)[matrix * p.out_sb + r * p.out_sr + c] = from_f32<T>(f[c & 3]);
        }
      __syncthreads();
    }
  }
  if (s_gave_up) {
    const unsigned long long until = device_ns() + 20000000ull;
    while (device_ns() < until) {}
  }
  __syncthreads();
  if (warp == 0) tmem_free<1>(tmem, p.columns);
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------

int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }  // rows on 16 bytes

// Scratch memory of a call: a batch is worked on `nb` matrices at a time.
struct Layout {
  int m, n;
  bool flip;
  int64_t nb;
  int blocks;  // partial sums of squares a matrix
  uint64_t part, factors, scale, x[2], xt[2], a, b, bytes;
};

int64_t matrix_bytes(int64_t m, int64_t n) { return 2 * 2 * (2 * m * padded(n) + 2 * n * padded(m) + 2 * m * padded(m)); }

Layout layout_of(const mf_orthogonalize_args& p) {
  Layout l{};
  l.flip = p.rows > p.cols;
  l.m = (int)(l.flip ? p.cols : p.rows);
  l.n = (int)(l.flip ? p.rows : p.cols);
  // (at most 4 GB of scratch where a matrix needs less, and what the launches' grids hold)
  l.nb = (int64_t(4) << 30) / matrix_bytes(l.m, l.n);
  l.nb = l.nb < 1 ? 1 : l.nb > 16384 ? 16384 : l.nb;
  if (l.nb > p.batch) l.nb = p.batch;
  // (2048 values a thread's turn; several rows side by side where they are short)
  const int64_t turns = (p.rows * ((p.cols + 7) / 8) + 255) / 256;
  l.blocks = (int)(turns < 4 ? 1 : turns / 4 > 600 ? 600 : turns / 4);
  uint64_t at = 0;
  const auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at += (bytes + 1023) / 1024 * 1024;
    return here;
  };
  l.part = take(sizeof(Squares) * (uint64_t)l.nb * l.blocks);
  l.factors = take(sizeof(float2) * 3 * (uint64_t)p.steps * l.nb);
  l.scale = take(sizeof(Scale) * (uint64_t)l.nb);
  for (int i = 0; i < 2 && i < p.steps; ++i) {  // (the last step's result is the call's)
    l.x[i] = take(4 * (uint64_t)l.nb * l.m * padded(l.n));
    l.xt[i] = take(4 * (uint64_t)l.nb * l.n * padded(l.m));
  }
  if (p.steps) {
    l.a = take(4 * (uint64_t)l.nb * l.m * padded(l.m));
    l.b = take(4 * (uint64_t)l.nb * l.m * padded(l.m));
  }
  l.bytes = at + 1024;  // (the start is rounded up to 1 KB)
  return l;
}

// The tensor maps of a call: a matrix's map serves every step that uses its place with the same parts (encoding one takes
// the host about a microsecond; a call's 15 products use some 75, a fifth of them different).
struct MapCache {
  struct Key {
    const void* p;
    int parts, rows, cols, box_rows, box_cols, swizzle;
    bool operator==(const Key& k) const {
      return p == k.p && parts == k.parts && rows == k.rows && cols == k.cols && box_rows == k.box_rows && box_cols == k.box_cols &&
             swizzle == k.swizzle;
    }
  };
  static constexpr int kMost = 48;
  Key key[kMost];
  CUtensorMap map[kMost];
  int n = 0;
};

// A tensor map of a matrix of parts with boxes of box_rows rows of box_cols values.
mf_status parts_map(MapCache& cache, CUtensorMap* map, const Parts& x, int rows, int cols, int batch, int box_rows, int box_cols,
                    CUtensorMapSwizzle swizzle) {
  const MapCache::Key key{x.p, x.parts, rows, cols, box_rows, box_cols, (int)swizzle};
  for (int i = 0; i < cache.n; ++i)
    if (cache.key[i] == key) {
      *map = cache.map[i];
      return MF_OK;
    }
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch * x.parts};
  const cuuint64_t strides[2] = {(cuuint64_t)x.ld * 2, (cuuint64_t)x.matrix * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
  if (!tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, x.p, dims, strides, box, swizzle)) {
    set_error("mf_orthogonalize: the driver refuses a tensor map");
    return MF_ECUDA;
  }
  if (cache.n < MapCache::kMost) {
    cache.key[cache.n] = key;
    cache.map[cache.n++] = *map;
  }
  return MF_OK;
}

template <int CTAS, int BN, int BK, int EPI, typename T>
mf_status launch_product(const Product& p, const Parts& a, const Parts& b, MapCache& cache, int sms, cudaStream_t s) {
  const auto kernel = k_orth_mma<CTAS, BN, BK, EPI, T>;
  constexpr CUtensorMapSwizzle kOperand = BK == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
  MmaMaps maps{};
  mf_status st = parts_map(cache, &maps.a, a, p.rows, p.depth, p.batch, kTileM, BK, kOperand);
  if (st == MF_OK) st = parts_map(cache, &maps.b, b, p.cols, p.depth, p.batch, BN / CTAS, BK, kOperand);
  if (st == MF_OK && EPI != kGram) st = parts_map(cache, &maps.old, p.old, p.rows, p.cols, p.batch, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
  if (st == MF_OK && EPI != kFinal) st = parts_map(cache, &maps.out, p.out, p.rows, p.cols, p.batch, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
  if (st == MF_OK && EPI != kFinal) st = parts_map(cache, &maps.out_t, p.out_t, p.cols, p.rows, p.batch, 32, 32, CU_TENSOR_MAP_SWIZZLE_NONE);
  if (st != MF_OK) return st;
  MF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_of(CTAS, BN, BK, EPI)));
  const int cluster = CTAS == 2 ? 2 : p.splits;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(sms / cluster * cluster));
  cfg.blockDim = dim3(mma_threads(CTAS, BK));
  cfg.dynamicSmemBytes = shared_of(CTAS, BN, BK, EPI);
  cfg.stream = s;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  int groups = sms;  // blocks or pairs that walk the tiles: as many as fit at once (not every SM of a GPC finds a partner)
  if (CTAS == 2) {
    static std::atomic<int> pairs[16];  // of each device, once its driver has said so
    int dev = 0, n = 0;
    MF_CUDA(cudaGetDevice(&dev));
    if (dev < 16) n = pairs[dev].load(std::memory_order_relaxed);
    if (!n) {
      MF_CUDA(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
      if (dev < 16) pairs[dev].store(n, std::memory_order_relaxed);
    }
    if (n < 1) {
      set_error("mf_orthogonalize: no pair of blocks fits the device");
      return MF_EUNSUPPORTED;
    }
    groups = n;
  }
  if (p.splits > 1 || p.tiles < groups) groups = p.tiles;
  cfg.gridDim = dim3((unsigned)(groups * cluster));
  MF_CUDA(cudaLaunchKernelEx(&cfg, kernel, p, maps));
  return MF_OK;
}

// Tiles of tm x bn of a matrix's result that are computed.
int tiles_of(const Product& p, int tm, int bn, int* rows, int* cols) {
  *rows = (p.rows + tm - 1) / tm;
  *cols = (p.cols + bn - 1) / bn;
  if (!p.symmetric) return *rows * *cols;
  int n = 0;
  for (int r = 0; r < *rows; ++r) {
    const int reach = (r * tm + tm - 1) / bn + 1;
    n += reach < *cols ? reach : *cols;
  }
  return n;
}

// Which tiles: pairs of SMs on 256 x 256 where these fill the GPU, else 128 x 128 or 128 x 64 on one, with the depth split
// over up to 8 blocks while SMs are idle.  By an estimate in cycles: a round of tiles takes its products (16 deep:
// 128 for a pair, whose SMs are then bound by the tensor cores, 80 and 75 for the others, bound by shared memory), the
// last tile's blocks (about 700 each), 1000 + 700 n for a cluster of n, and 3000 for the start.
template <int EPI, typename T>
mf_status product(Product p, const Parts& a, const Parts& b, MapCache& cache, int sms, cudaStream_t s) {
  p.na = a.parts;
  p.nb = b.parts;
  const int terms = a.parts + b.parts - 1;
  const int64_t steps = (p.depth + 15) / 16 * terms;
  const bool split = a.parts > 1 || b.parts > 1 || p.depth > kLongSum;  // (stages of 32, sums in parts)
  const int stages = (p.depth + (split ? 31 : 63)) / (split ? 32 : 64);
  struct Shape { int ctas, bn, cycles; };
  const Shape shapes[3] = {{2, 256, 128}, {1, 128, 80}, {1, 64, 75}};
  int best = 0, best_splits = 1;
  double least = 1e300;
  for (int i = 0; i < 3; ++i) {
    const Shape& h = shapes[i];
    int r, c;
    const int64_t tiles = (int64_t)tiles_of(p, 128 * h.ctas, h.bn, &r, &c) * p.batch;
    for (int n = 1; n <= (h.ctas == 2 ? 1 : 8) && n <= stages; n *= 2) {
      const int64_t at_once = sms / (h.ctas * n);
      const int64_t rounds = (tiles + at_once - 1) / at_once;
      if (n > 1 && rounds > 1) break;
      const double t = (double)rounds * steps * h.cycles / n + h.bn / 32 * 700.0 / n + (n > 1 ? 1000.0 + 700.0 * n : 0.0) + 3000.0;
      if (t < least) {
        least = t;
        best = i;
        best_splits = n;
      }
    }
  }
  p.splits = best_splits;
  const int64_t tiles = (int64_t)tiles_of(p, 128 * shapes[best].ctas, shapes[best].bn, &p.tiles_r, &p.tiles_c) * p.batch;
  if (tiles > (1 << 30)) {
    set_error("mf_orthogonalize: the matrices have too many tiles");
    return MF_EUNSUPPORTED;
  }
  p.tiles = (int)tiles;
  if (best == 0) return split ? launch_product<2, 256, 32, EPI, T>(p, a, b, cache, sms, s) : launch_product<2, 256, 64, EPI, T>(p, a, b, cache, sms, s);
  if (best == 1) return split ? launch_product<1, 128, 32, EPI, T>(p, a, b, cache, sms, s) : launch_product<1, 128, 64, EPI, T>(p, a, b, cache, sms, s);
  return split ? launch_product<1, 64, 32, EPI, T>(p, a, b, cache, sms, s) : launch_product<1, 64, 64, EPI, T>(p, a, b, cache, sms, s);
}

// The steps' factors: operands are X sx, A sa and B sb.  (Step 0: its operands times rho / sx are X, which factors_of puts in.)
void steps_of(const mf_orthogonalize_args& p, Steps* out) {
  const auto scale_below = [](double top) { return std::ldexp(1.0, scale_exp((float)top)); };
  // parts of step k's operands: see the comment at the top and mf.h
  const auto parts_of = [&](int k) { return p.type == MF_TYPE_BF16 && k >= p.steps - 2 ? 1 : 2; };
  double top = 1.0, sx = 1.0;
  out->n = p.steps;
  out->a = p.a;
  out->b = p.b;
  out->c = p.c;
  for (int k = 0; k < p.steps; ++k) {
    const double most = orth_largest(p, top);
    const double most_b = std::fabs(p.b) * top * top + std::fabs(p.c) * top * top * top * top;
    // (a tenth more for what roundings add)
    const double sa = scale_below(1.1 * top * top), sb = scale_below(1.1 * most_b);
    const bool end = k + 1 == p.steps;
    const double sx1 = end ? 1.0 : scale_below(1.1 * most);
    Step& t = out->step[k];
    t.top = (float)(1.001 * top);
    t.parts = parts_of(k);
    t.next_parts = end ? 0 : parts_of(k + 1);
    t.f.gram = (float)(sa / (sx * sx));
    t.f.square_acc = (float)(p.c * sb / (sa * sa));
    t.f.square_old = (float)(p.b * sb / sa);
    t.f.apply_acc = (float)(sx1 / (sb * sx));
    t.f.apply_old = (float)(p.a * sx1 / sx);
    top = most;
    sx = sx1;
  }
}

// Whether a matrix's operands fit a block's shared memory (and its sums tensor memory); fills the layout.
constexpr uint32_t kSmallShared = 224u << 10;
bool small_layout(const mf_orthogonalize_args& p, Small* q, uint32_t* bytes) {
  const bool flip = p.rows > p.cols;
  const int64_t m = flip ? p.cols : p.rows, n = flip ? p.rows : p.cols;
  if (p.steps == 0 || m > 128 || n > 512) return false;
  q->m = (int)m;
  q->n = (int)n;
  q->flip = flip;
  q->mp = (q->m + 15) / 16 * 16;
  q->np = (q->n + 15) / 16 * 16;
  q->ap = (uint32_t)((q->mp + 63) / 64 * q->mp * 128);
  q->xp = (uint32_t)((q->np + 63) / 64 * q->mp * 128);
  q->tp = (uint32_t)((q->mp + 63) / 64 * q->np * 128);
  q->xoff = 2 * q->ap;
  q->toff = q->xoff + 2 * q->xp;
  uint32_t end = q->toff + 2 * q->tp;
  // (a product reads 128 rows of its first operand, A or X, whatever they hold)
  const uint32_t reach = q->toff + (128 - q->mp) * 128;
  if (end < reach) end = reach;
  *bytes = end + 1024;
  q->columns = 32;
  while ((int)q->columns < q->np || (int)q->columns < q->mp) q->columns *= 2;
  q->cross = q->columns <= 256 ? q->columns : 0;
  q->columns += q->cross;
  return *bytes <= kSmallShared;
}

template <typename T>
mf_status run_small(const mf_orthogonalize_args& p, Small& q, uint32_t bytes, const Waits& waits, cudaStream_t s) {
  int dev = 0, sms = 0, per_sm = 0;
  MF_CUDA(cudaGetDevice(&dev));
  MF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  q.in = {p.d_g, p.g_stride_batch, p.g_stride_row, (int)p.rows, (int)p.cols};
  q.out = p.d_out;
  q.out_sb = p.out_stride_batch;
  q.out_sr = p.out_stride_row;
  q.batch = p.batch;
  q.eps = p.eps;
  q.waits = waits;
  steps_of(p, &q.steps);
  q.first_parts = sizeof(T) == 2 ? 1 : q.steps.step[0].parts;
  MF_CUDA(cudaFuncSetAttribute(k_orth_small<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallShared));
  // as many blocks an SM as shared memory, threads and tensor memory hold
  per_sm = (int)(kSmallShared / bytes);
  if (per_sm > 512 / (int)q.columns) per_sm = 512 / (int)q.columns;
  if (per_sm > 2) per_sm = 2;
  if (per_sm < 1) per_sm = 1;
  const int64_t most = (int64_t)sms * per_sm;
  k_orth_small<T><<<(unsigned)(p.batch < most ? p.batch : most), kSmallThreads, bytes, s>>>(q);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

template <typename T>
mf_status run(const mf_orthogonalize_args& p, char* work, const Waits& waits, cudaStream_t s) {
  Small small{};
  uint32_t bytes = 0;
  if (small_layout(p, &small, &bytes)) return run_small<T>(p, small, bytes, waits, s);
  const Layout l = layout_of(p);
  work += (1024 - ((uintptr_t)work & 1023)) & 1023;
  int dev = 0, sms = 0;
  MF_CUDA(cudaGetDevice(&dev));
  MF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int m = l.m, n = l.n;
  Steps steps;
  steps_of(p, &steps);
  for (int64_t b0 = 0; b0 < p.batch; b0 += l.nb) {
    const int nb = (int)(p.batch - b0 < l.nb ? p.batch - b0 : l.nb);
    const Input in{(const T*)p.d_g + b0 * p.g_stride_batch, p.g_stride_batch, p.g_stride_row, (int)p.rows, (int)p.cols};
    T* out = (T*)p.d_out + b0 * p.out_stride_batch;
    Squares* part = (Squares*)(work + l.part);
    float2* factors = (float2*)(work + l.factors);
    Scale* scale = (Scale*)(work + l.scale);
    k_orth_squares<T><<<dim3(l.blocks, nb), 256, 0, s>>>(in, part);
    k_orth_scale<<<nb, 32, 0, s>>>(part, l.blocks, p.eps, steps, scale, factors);
    if (p.steps == 0) {
      k_orth_scaled<T><<<dim3(l.blocks, nb), 256, 0, s>>>(in, scale, out, p.out_stride_batch, p.out_stride_row);
      MF_CUDA(cudaGetLastError());
      continue;
    }
    const auto matrix = [&](uint64_t at, int rows, int cols, int parts) {
      return Parts{(__half*)(work + at), padded(cols), rows * padded(cols), nb * rows * padded(cols), parts};
    };
    // (16-bit values are operands of one part as they are)
    const int first_parts = sizeof(T) == 2 ? 1 : steps.step[0].parts;
    Parts x = matrix(l.x[0], m, n, first_parts), xt = matrix(l.xt[0], n, m, first_parts);
    k_orth_first<T><<<dim3((in.cols + 63) / 64, (in.rows + 63) / 64, nb), 256, 0, s>>>(in, scale, l.flip, x, xt);
    MF_CUDA(cudaGetLastError());
    MapCache cache;
    for (int k = 0; k < p.steps; ++k) {
      const Step& t = steps.step[k];
      const int parts = t.parts;
      const Parts a = matrix(l.a, m, m, parts), b = matrix(l.b, m, m, parts);
      Product q{};
      q.batch = nb;
      q.waits = waits;
      q.rows = q.cols = m;
      q.symmetric = true;
      q.depth = n;
      q.chunk = chunk_of(p.type, n);
      q.factors = factors + (int64_t)k * 3 * nb;
      q.out = q.out_t = a;
      mf_status st = product<kGram, float>(q, x, x, cache, sms, s);
      q.depth = m;
      q.chunk = chunk_of(p.type, m);
      q.factors += nb;
      q.old = a;
      q.out = q.out_t = b;
      if (st == MF_OK) st = product<kSquare, float>(q, a, a, cache, sms, s);
      q.symmetric = false;
      q.cols = n;
      q.factors += nb;
      q.old = x;
      if (k + 1 < p.steps) {
        const Parts y = matrix(l.x[(k + 1) & 1], m, n, t.next_parts), yt = matrix(l.xt[(k + 1) & 1], n, m, t.next_parts);
        q.out = y;
        q.out_t = yt;
        if (st == MF_OK) st = product<kApply, float>(q, b, xt, cache, sms, s);
        x = y;
        xt = yt;
      } else {
        q.final_out = out;
        q.final_sb = p.out_stride_batch;
        q.final_sr = p.out_stride_row;
        q.flip = l.flip;
        if (st == MF_OK) st = product<kFinal, T>(q, b, xt, cache, sms, s);
      }
      if (st != MF_OK) return st;
    }
  }
  return MF_OK;
}

}  // namespace

double orth_largest(const mf_orthogonalize_args& p, double top) {
  const double a = p.a, b = p.b, c = p.c;
  const auto size = [&](double t) { return std::sqrt(t) * std::fabs(a + t * (b + t * c)); };  // t = s^2
  double most = size(top * top);
  // 5 c t^2 + 3 b t + a = 0
  double roots[2] = {-1.0, -1.0};
  if (c == 0.0) {
    if (b != 0.0) roots[0] = -a / (3.0 * b);
  } else if (const double d = 9.0 * b * b - 20.0 * a * c; d >= 0.0) {
    roots[0] = (-3.0 * b + std::sqrt(d)) / (10.0 * c);
    roots[1] = (-3.0 * b - std::sqrt(d)) / (10.0 * c);
  }
  for (const double t : roots)
    if (t > 0.0 && t < top * top && size(t) > most) most = size(t);
  return most;
}

mf_status orth_work(const mf_orthogonalize_args& p, uint64_t* bytes) {
  Small small{};
  uint32_t shared = 0;
  *bytes = small_layout(p, &small, &shared) ? 0 : layout_of(p).bytes;
  return MF_OK;
}

mf_status orth_run(const mf_orthogonalize_args& p, void* work, uint32_t wait_test, cudaStream_t s) {
  const Waits waits{wait_test, wait_test ? 16u : 0u, p.d_status};
  if (p.type == MF_TYPE_F32) return run<float>(p, (char*)work, waits, s);
  if (p.type == MF_TYPE_BF16) return run<__nv_bfloat16>(p, (char*)work, waits, s);
  return run<__half>(p, (char*)work, waits, s);
}

}  // namespace mf
