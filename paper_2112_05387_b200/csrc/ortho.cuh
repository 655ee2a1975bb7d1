// Orthogonalised update: kernels around the products of gemm_tc.cuh.
//
//   X_0 = G / max(|G|_F, eps);   X <- a X + b (X X^T) X + c (X X^T)^2 X,   `steps` times
// computed as A = X X^T, B = a I + b A + c A^2, X <- B X on the smaller side (X^T X and X B for tall matrices).
//
// Two passes over G come before the products: the Frobenius norm (with the momentum, where there is one), and the fp16
// planes of G 2^k, k chosen so that the norm lies in [2^14, 2^15).  G's scale is not divided out here: alpha = 1 / (norm 2^k)
// goes into the first products' epilogues, so a bf16 gradient enters the iteration without a rounding (8 significant bits
// fit fp16's 11; elements more than 2^32 below the norm keep fewer).
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "gemm_tc.cuh"

namespace lp {

constexpr int kOrthoThreads = 256;
constexpr int kOrthoMaxParts = 512;

struct OrthoSource {
  const void* g;          // gradients, fp32 or bf16, contiguous matrices
  int g_bf16;
  float* momentum;        // null: G itself is orthogonalised
  float mu;
  int nesterov;
  long long elems;        // of one matrix
  int use_off;
  long long off[tc::kGemmMaxOffsets];
};

__device__ __forceinline__ float ortho_grad(const OrthoSource& s, long long i) {
  return s.g_bf16 ? __bfloat162float(((const bf16*)s.g)[i]) : ((const float*)s.g)[i];
}

// Sums of squares of what is orthogonalised, `parts` partial sums a matrix; the momentum is updated on the way:
//   m <- mu m + g;  u = m, or g + mu m (Nesterov).
__global__ void __launch_bounds__(kOrthoThreads)
ortho_norm_kernel(const __grid_constant__ OrthoSource s, int parts, double* __restrict__ sums, int* __restrict__ err) {
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *err = 0;
  const int b = blockIdx.y;
  const long long base = s.use_off ? s.off[b] : b * s.elems;
  const long long lo = s.elems * blockIdx.x / parts, hi = s.elems * (blockIdx.x + 1) / parts;
  double sum = 0.0;
#pragma unroll 4
  for (long long i = lo + threadIdx.x; i < hi; i += kOrthoThreads) {
    float u = ortho_grad(s, base + i);
    if (s.momentum) {
      const float g = u;
      const float m = fmaf(s.mu, s.momentum[base + i], g);
      s.momentum[base + i] = m;
      u = s.nesterov ? fmaf(s.mu, m, g) : m;
    }
    sum += (double)u * (double)u;
  }
  __shared__ double part[kOrthoThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kOrthoThreads / 32; ++w) sum += part[w];
    sums[(long long)b * parts + blockIdx.x] = sum;
  }
}

// fp16 planes of u 2^k (rows `ld` apart), and alpha = 1 / (max(norm, eps) 2^k) of each matrix.
__global__ void __launch_bounds__(kOrthoThreads)
ortho_pack_kernel(const __grid_constant__ OrthoSource s, int parts, const double* __restrict__ sums, float eps, int cols, long long ld,
                  __half* __restrict__ x, long long x_batch, long long x_plane /* 0: no low part */, float* __restrict__ alpha) {
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.y;
  __shared__ float scale_s;
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 32) sum += sums[(long long)b * parts + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x == 0) {
      const double norm = fmax(sqrt(sum), (double)eps);
      const int k = isfinite(norm) ? 14 - ilogb(norm) : 0;
      scale_s = (float)ldexp(1.0, k);
      if (blockIdx.x == 0) alpha[b] = (float)(1.0 / ldexp(norm, k));
    }
  }
  __syncthreads();
  const float scale = scale_s;
  const long long base = s.use_off ? s.off[b] : b * s.elems;
  __half* out = x + b * x_batch;
  for (long long i = (long long)blockIdx.x * kOrthoThreads + threadIdx.x; i < s.elems; i += (long long)gridDim.x * kOrthoThreads) {
    float u = ortho_grad(s, base + i);
    if (s.momentum) {
      const float m = s.momentum[base + i];
      u = s.nesterov ? fmaf(s.mu, m, u) : m;
    }
    __half hi, lo;
    tc::split_half(u * scale, hi, lo);
    const long long r = i / cols, at = r * ld + (i - r * cols);
    out[at] = hi;
    if (x_plane) out[x_plane + at] = lo;
  }
}

}  // namespace lp
