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
constexpr int kOrthoMaxParts = 1184;

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

// kVec: eight elements at a time (matrices start on a multiple of 8 elements), else one.
template <bool kVec>
struct OrthoVec {
  static constexpr int N = kVec ? 8 : 1;
};
template <bool kVec>
__device__ __forceinline__ void ortho_load(const void* p, int is_bf16, long long i, float (&v)[OrthoVec<kVec>::N]) {
  if constexpr (kVec) {
    if (is_bf16) {
      ldv((const bf16*)p + i, v);
    } else {
      float a[4], b[4];
      ldv((const float*)p + i, a);
      ldv((const float*)p + i + 4, b);
#pragma unroll
      for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[4 + j] = b[j]; }
    }
  } else {
    v[0] = is_bf16 ? __bfloat162float(((const bf16*)p)[i]) : ((const float*)p)[i];
  }
}
template <bool kVec>
__device__ __forceinline__ void ortho_store(float* p, long long i, const float (&v)[OrthoVec<kVec>::N]) {
  if constexpr (kVec) {
    *reinterpret_cast<float4*>(p + i) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    p[i] = v[0];
  }
}
// What is orthogonalised, from the gradient and the momentum after its update.
template <int N>
__device__ __forceinline__ void ortho_direction(const OrthoSource& s, float (&g)[N], const float (&m)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) g[j] = s.nesterov ? fmaf(s.mu, m[j], g[j]) : m[j];
}

// Updates the momentum of a group (if there is one); the sum of squares of what is orthogonalised.
template <bool kVec>
__device__ __forceinline__ double ortho_square(const OrthoSource& s, long long i) {
  constexpr int N = OrthoVec<kVec>::N;
  float u[N];
  ortho_load<kVec>(s.g, s.g_bf16, i, u);
  if (s.momentum) {
    float m[N];
    ortho_load<kVec>(s.momentum, 0, i, m);
#pragma unroll
    for (int j = 0; j < N; ++j) m[j] = fmaf(s.mu, m[j], u[j]);
    ortho_store<kVec>(s.momentum, i, m);
    ortho_direction(s, u, m);
  }
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j) sum += (double)u[j] * (double)u[j];
  return sum;
}

// Sums of squares of what is orthogonalised, `parts` partial sums a matrix, in fp64 (a gradient of 1e-25 or 1e25 squares out of
// fp32's range); the momentum is updated on the way:
//   m <- mu m + g;  u = m, or g + mu m (Nesterov).
template <bool kVec>
__global__ void __launch_bounds__(kOrthoThreads)
ortho_norm_kernel(const __grid_constant__ OrthoSource s, int parts, double* __restrict__ sums, int* __restrict__ err /* cleared, or null */) {
  constexpr int N = OrthoVec<kVec>::N;
  pdl_wait();
  pdl_launch_dependents();
  if (err && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *err = 0;
  const int b = blockIdx.y;
  const long long base = s.use_off ? s.off[b] : b * s.elems, groups = s.elems / N;
  const long long lo = groups * blockIdx.x / parts, hi = groups * (blockIdx.x + 1) / parts;
  double sum = 0.0;
#pragma unroll 2
  for (long long i = lo + threadIdx.x; i < hi; i += kOrthoThreads) sum += ortho_square<kVec>(s, base + i * N);
  // (what is left of a matrix that does not end on a group)
  if (kVec && blockIdx.x == 0 && threadIdx.x < s.elems - groups * N) sum += ortho_square<false>(s, base + groups * N + threadIdx.x);
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

// Scale 2^k of a matrix's planes and alpha = 1 / (max(norm, eps) 2^k), from the partial sums of squares; by one warp.
__device__ __forceinline__ void ortho_scale(const double* sums, int parts, float eps, float& scale, float& alpha) {
  double sum = 0.0;
  for (int i = threadIdx.x & 31; i < parts; i += 32) sum += sums[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const double norm = fmax(sqrt(sum), (double)eps);
  const int k = isfinite(norm) ? 14 - ilogb(norm) : 0;
  scale = (float)ldexp(1.0, k);
  alpha = (float)(1.0 / ldexp(norm, k));
}

// fp16 planes of u 2^k (rows `ld` apart, padded to whole groups of 8), and alpha.  A thread has 8 columns of a row; where rows do
// not start on a group (kVec false) it reads them one by one.
template <bool kVec>
__global__ void __launch_bounds__(kOrthoThreads)
ortho_pack_kernel(const __grid_constant__ OrthoSource s, int parts, const double* __restrict__ sums, float eps, int cols, long long ld,
                  __half* __restrict__ x, long long x_batch, long long x_plane /* 0: no low part */, float* __restrict__ alpha) {
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.y;
  __shared__ float scale_s;
  if (threadIdx.x < 32) {
    float sc, al;
    ortho_scale(sums + (long long)b * parts, parts, eps, sc, al);
    if (threadIdx.x == 0) {
      scale_s = sc;
      if (blockIdx.x == 0) alpha[b] = al;
    }
  }
  __syncthreads();
  const float scale = scale_s;
  const long long base = s.use_off ? s.off[b] : b * s.elems;
  const int per_row = (cols + 7) / 8;
  const long long groups = s.elems / cols * per_row;
  __half* out = x + b * x_batch;
#pragma unroll 2
  for (long long i = (long long)blockIdx.x * kOrthoThreads + threadIdx.x; i < groups; i += (long long)gridDim.x * kOrthoThreads) {
    // (a 64-bit division costs as much as the rest of the loop)
    const long long r = groups >> 32 ? i / per_row : (long long)((uint32_t)i / (uint32_t)per_row);
    const int c = (int)(i - r * per_row) * 8;
    const long long from = base + r * cols + c;
    float u[8], m[8];
    if constexpr (kVec) {
      ortho_load<true>(s.g, s.g_bf16, from, u);
      if (s.momentum) ortho_load<true>(s.momentum, 0, from, m);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float a[1] = {0.f};
        if (c + j < cols) ortho_load<false>(s.g, s.g_bf16, from + j, a);
        u[j] = a[0];
        m[j] = s.momentum && c + j < cols ? s.momentum[from + j] : 0.f;
      }
    }
    if (s.momentum) ortho_direction(s, u, m);
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) tc::split_f16x2(u[2 * j] * scale, u[2 * j + 1] * scale, hi[j], lo[j]);
    __half* at = out + r * ld + c;
    *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (x_plane) *reinterpret_cast<uint4*>(at + x_plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

}  // namespace lp
