// Orthogonalisation of matrices by Newton-Schulz products (the operators' section of include/mf.h).
#include "mf_ops.cuh"

namespace mf {
namespace {

// A matrix's squares in three ranges, so that none overflows or underflows in fp32: small values
// scaled by 2^96, large ones by 2^-80 (each sum then stays far inside the range).
struct Squares {
  float mid = 0.f, small = 0.f, large = 0.f;
  __device__ __forceinline__ void add(float v) {
    const float m = fabsf(v);
    if (m < 0x1p-48f) small = fmaf(v * 0x1p96f, v * 0x1p96f, small);
    else if (m > 0x1p48f) large = fmaf(v * 0x1p-80f, v * 0x1p-80f, large);
    else mid = fmaf(v, v, mid);  // (NaN too)
  }
  __device__ __forceinline__ double total() const {
    return (double)mid + (double)small * 0x1p-192 + (double)large * 0x1p160;
  }
};

// Three factors whose product is 1 / (norm + eps), each a normal fp32 number: two powers of two, and a
// rest in (1/2, 1].
__device__ __forceinline__ void inverse_parts(double sum, float eps, float (&r)[3]) {
  const double n = sqrt(sum) + (double)eps;
  if (n == 0.0) { r[0] = r[1] = r[2] = 1.f; return; }  // (zeros stay zeros)
  if (!isfinite(n)) { r[0] = r[1] = r[2] = __int_as_float(0x7fc00000); return; }
  int e;
  const double f = frexp(n, &e);  // n = f 2^e, f in [1/2, 1)
  r[0] = ldexpf(1.f, -(e / 2));
  r[1] = ldexpf(1.f, -(e - e / 2) + 1);
  r[2] = (float)(0.5 / f);
}

template <typename T>
__global__ void __launch_bounds__(1024) k_orth_start(const T* g, int64_t sb, int64_t sr, int rows, int cols, float eps,
                                                     float* x, bool flip) {
  __shared__ double part[1024];
  const T* p = g + blockIdx.x * sb;
  const int64_t n = (int64_t)rows * cols;
  Squares q;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) q.add(to_f32(p[i / cols * sr + i % cols]));
  part[threadIdx.x] = q.total();
  __syncthreads();
  for (int w = 512; w > 0; w >>= 1) {
    if (threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
    __syncthreads();
  }
  float r[3];
  inverse_parts(part[0], eps, r);
  x += blockIdx.x * n;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) {
    const int64_t row = i / cols, col = i % cols;
    x[flip ? col * rows + row : i] = to_f32(p[row * sr + col]) * r[0] * r[1] * r[2];
  }
}

// D = alpha E + beta P Q (row-major, P m x k, Q k x n or its transpose), 64 x 64 tiles.
struct Product {
  const float *p, *q, *e;
  float* d;
  int m, n, k, qt;
  float alpha, beta;
};
__global__ void __launch_bounds__(256) k_orth_product(const Product a) {
  __shared__ float sp[16][65], sq[16][65];
  const int64_t b = blockIdx.z;
  const float* p = a.p + b * a.m * a.k;
  const float* q = a.q + b * a.n * a.k;
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, tr = threadIdx.x / 16 * 4, tc = threadIdx.x % 16 * 4;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < a.k; k0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int kk = i % 16, r = i / 16;
      sp[kk][r] = r0 + r < a.m && k0 + kk < a.k ? p[(int64_t)(r0 + r) * a.k + k0 + kk] : 0.f;
      if (a.qt) {
        sq[kk][r] = c0 + r < a.n && k0 + kk < a.k ? q[(int64_t)(c0 + r) * a.k + k0 + kk] : 0.f;
      } else {
        const int c = i % 64, kr = i / 64;
        sq[kr][c] = c0 + c < a.n && k0 + kr < a.k ? q[(int64_t)(k0 + kr) * a.n + c0 + c] : 0.f;
      }
    }
    __syncthreads();
    for (int kk = 0; kk < 16; ++kk)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sp[kk][tr + i], sq[kk][tc + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j)
      if (r0 + tr + i < a.m && c0 + tc + j < a.n) {
        const int64_t at = (b * a.m + r0 + tr + i) * a.n + c0 + tc + j;
        a.d[at] = a.beta * acc[i][j] + (a.e ? a.alpha * a.e[at] : 0.f);
      }
}

template <typename T>
__global__ void k_orth_end(const float* x, T* out, int64_t sb, int64_t sr, int64_t rows, int64_t cols, bool flip) {
  const int64_t n = rows * cols;
  x += blockIdx.y * n;
  out += blockIdx.y * sb;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t row = i / cols, col = i % cols;
    out[row * sr + col] = from_f32<T>(x[flip ? col * rows + row : i]);
  }
}

template <typename T>
mf_status run(const mf_orthogonalize_args& p, float* work, cudaStream_t s) {
  const bool flip = p.rows > p.cols;
  const int m = (int)(flip ? p.cols : p.rows), n = (int)(flip ? p.rows : p.cols);
  const int64_t most = 32768;  // matrices a launch (grid limit)
  for (int64_t b0 = 0; b0 < p.batch; b0 += most) {
    const unsigned nb = (unsigned)(p.batch - b0 < most ? p.batch - b0 : most);
    float *x = work, *y = x + (int64_t)nb * m * n, *A = y + (int64_t)nb * m * n, *B = A + (int64_t)nb * m * m;
    const dim3 gx((n + 63) / 64, (m + 63) / 64, nb), ga((m + 63) / 64, (m + 63) / 64, nb);
    k_orth_start<T><<<nb, 1024, 0, s>>>((const T*)p.d_g + b0 * p.g_stride_batch, p.g_stride_batch, p.g_stride_row, (int)p.rows,
                                        (int)p.cols, p.eps, x, flip);
    for (int i = 0; i < p.steps; ++i) {
      k_orth_product<<<ga, 256, 0, s>>>(Product{x, x, nullptr, A, m, m, n, 1, 0.f, 1.f});
      k_orth_product<<<ga, 256, 0, s>>>(Product{A, A, A, B, m, m, m, 0, p.b, p.c});
      k_orth_product<<<gx, 256, 0, s>>>(Product{B, x, x, y, m, n, m, 0, p.a, 1.f});
      float* t = x; x = y; y = t;
    }
    k_orth_end<T><<<dim3(256, nb), 256, 0, s>>>(x, (T*)p.d_out + b0 * p.out_stride_batch, p.out_stride_batch, p.out_stride_row,
                                                p.rows, p.cols, flip);
    MF_CUDA(cudaGetLastError());
  }
  return MF_OK;
}

}  // namespace

mf_status orth_work(const mf_orthogonalize_args& p, uint64_t* bytes) {
  const uint64_t m = (uint64_t)(p.rows < p.cols ? p.rows : p.cols), n = (uint64_t)(p.rows < p.cols ? p.cols : p.rows);
  const uint64_t nb = (uint64_t)(p.batch < 32768 ? p.batch : 32768);
  *bytes = 4 * nb * (2 * m * n + 2 * m * m);
  return MF_OK;
}

mf_status orth_run(const mf_orthogonalize_args& p, void* work, cudaStream_t s) {
  if (p.type == MF_TYPE_F32) return run<float>(p, (float*)work, s);
  if (p.type == MF_TYPE_BF16) return run<__nv_bfloat16>(p, (float*)work, s);
  return run<__half>(p, (float*)work, s);
}

}  // namespace mf
