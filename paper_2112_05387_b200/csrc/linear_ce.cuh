// Softmax cross entropy of a linear layer over many classes: kernels around the products of gemm_tc.cuh.
//
//   l = x w^T + bias;  lse_t = log sum_v exp l_tv;  loss = mean over counted rows of lse_t - l_t,label
//   dl = g (softmax(l) - onehot) / count,  dx = dl w,  dw = dl^T x,  dbias = sum_t dl
//
// The logits are never stored.  The product's epilogue turns a tile of them into exponentials relative to the maximum of the
// row's part of the tile, and that maximum and the sum; the loss alone needs nothing else.  For the gradients the exponentials
// of a piece of the rows are kept in 16 bits, rescaled in place into dl once the rows' lse is known, and multiplied twice.
// Pieces of rows and not of classes: with the classes in pieces every logit would be computed twice (8 T D V operations
// instead of 6 T D V).
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "gemm_tc.cuh"

namespace lp {

constexpr int kCeThreads = 256;
constexpr float kCeDlScale = 16384.f;   // fp16 planes of dl (fp32 problems) hold dl times this: |dl| <= 1

// Device-side scalars at the start of the scratch.
struct CeHeader {
  int err;
  int count;          // rows whose label is a class
  float logit_f;      // scale of x w^T's accumulator
  float dx_f, dw_f;   // scales of the gradients' accumulators
  float x_scale, w_scale;
  float grad_f;       // g / count
};

__device__ __forceinline__ bool ce_counts(int label, int V) { return label >= 0 && label < V; }

__device__ __forceinline__ float block_sum(float v, float* part) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < kCeThreads / 32; ++i) s += part[i];
  __syncthreads();
  return s;
}

// Block 0 counts the rows; for fp32 problems the others take the largest finite magnitudes of x and w (parts of each).
__global__ void __launch_bounds__(kCeThreads)
ce_prepare_kernel(const int32_t* __restrict__ labels, int T, int V, const float* __restrict__ x, long long nx, const float* __restrict__ w,
                  long long nw, float* __restrict__ amax, int parts, CeHeader* __restrict__ hdr) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float part[kCeThreads / 32];
  if (blockIdx.x == 0) {
    int n = 0;
    for (int t = threadIdx.x; t < T; t += kCeThreads) n += ce_counts(labels[t], V);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    __shared__ int cnt[kCeThreads / 32];
    if ((threadIdx.x & 31) == 0) cnt[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int i = 1; i < kCeThreads / 32; ++i) n += cnt[i];
      hdr->err = 0;
      hdr->count = n;
    }
    return;
  }
  const int b = blockIdx.x - 1;
  const bool of_w = b >= parts;
  const float* v = of_w ? w : x;
  const long long n = of_w ? nw : nx;
  const int k = of_w ? b - parts : b;
  const long long lo = n * k / parts, hi = n * (k + 1) / parts;
  float m = 0.f;
#pragma unroll 4
  for (long long i = lo + threadIdx.x; i < hi; i += kCeThreads) {
    const float a = fabsf(v[i]);
    if (a <= 3.4028235e38f) m = fmaxf(m, a);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kCeThreads / 32; ++i) m = fmaxf(m, part[i]);
    amax[b] = m;
  }
}

// Power of two that takes `amax` into [2^14, 2^15).
__device__ __forceinline__ float ce_scale_of(float amax) {
  if (!(amax > 0.f)) return 1.f;
  const int e = 14 - ilogbf(amax);
  return ldexpf(1.f, e > 126 ? 126 : e);
}

// The operands as the products take them, rows `ld` apart: fp32 as fp16 high and low parts of the scaled values, bf16 as it is.
// Rows of x whose label is no class become zeros: what stands there (padding, NaN) must not reach dw through a product with 0.
// Blocks [0, xb) take x, the rest w (none where it is used in place).  The first block writes the header's scales.  kVec: D is a
// multiple of 8.
template <bool kVec>
__global__ void __launch_bounds__(kCeThreads)
ce_pack_kernel(const void* __restrict__ x, const void* __restrict__ w, const int32_t* __restrict__ labels, int is_bf16, int T, int D, int V,
               long long ld, __half* __restrict__ xo, long long x_plane, __half* __restrict__ wo, long long w_plane, int xb,
               const float* __restrict__ amax, int parts, float g, CeHeader* __restrict__ hdr) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float scales[2];
  if (threadIdx.x < 64) {
    const int which = threadIdx.x >> 5;
    float m = 0.f;
    if (!is_bf16)
      for (int i = threadIdx.x & 31; i < parts; i += 32) m = fmaxf(m, amax[which * parts + i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) scales[which] = is_bf16 ? 1.f : ce_scale_of(m);
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int n = hdr->count;
    const float gf = n > 0 ? g / (float)n : 0.f;
    const float dl = is_bf16 ? 1.f : 1.f / kCeDlScale;
    hdr->x_scale = scales[0];
    hdr->w_scale = scales[1];
    hdr->logit_f = (1.f / scales[0]) * (1.f / scales[1]);
    hdr->grad_f = gf;
    hdr->dx_f = gf * dl * (1.f / scales[1]);
    hdr->dw_f = gf * dl * (1.f / scales[0]);
  }
  const bool of_w = (int)blockIdx.x >= xb;
  const int blk = of_w ? blockIdx.x - xb : blockIdx.x, blks = of_w ? gridDim.x - xb : xb;
  const void* src = of_w ? w : x;
  __half* dst = of_w ? wo : xo;
  const long long plane = of_w ? w_plane : x_plane;
  const float scale = scales[of_w];
  constexpr int N = kVec ? 8 : 1;
  const int per_row = D / N;
  const long long n = (long long)(of_w ? V : T) * per_row;
#pragma unroll 2
  for (long long i = (long long)blk * kCeThreads + threadIdx.x; i < n; i += (long long)blks * kCeThreads) {
    const long long r = n >> 32 ? i / per_row : (long long)((uint32_t)i / (uint32_t)per_row);
    const long long from = i * N, at = r * ld + (i - r * per_row) * N;
    const bool keep = of_w || ce_counts(labels[r], V);
    if (is_bf16) {
      if constexpr (kVec) {
        uint4 v = ld_raw((const bf16*)src + from);
        if (!keep) v = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>((bf16*)dst + at) = v;
      } else {
        ((bf16*)dst)[at] = keep ? ((const bf16*)src)[from] : __float2bfloat16_rn(0.f);
      }
    } else {
      __half hi[N], lo[N];
      float v[N];
      if constexpr (kVec) {
        float a[4], b[4];
        ldv((const float*)src + from, a);
        ldv((const float*)src + from + 4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[4 + j] = b[j]; }
      } else {
        v[0] = ((const float*)src)[from];
      }
#pragma unroll
      for (int j = 0; j < N; ++j) tc::split_half(keep ? v[j] * scale : 0.f, hi[j], lo[j]);
      if constexpr (kVec) {
        *reinterpret_cast<uint4*>(dst + at) = make_uint4(tc::pack_half2(hi[0], hi[1]), tc::pack_half2(hi[2], hi[3]),
                                                         tc::pack_half2(hi[4], hi[5]), tc::pack_half2(hi[6], hi[7]));
        *reinterpret_cast<uint4*>(dst + plane + at) = make_uint4(tc::pack_half2(lo[0], lo[1]), tc::pack_half2(lo[2], lo[3]),
                                                                 tc::pack_half2(lo[4], lo[5]), tc::pack_half2(lo[6], lo[7]));
      } else {
        dst[at] = hi[0];
        dst[plane + at] = lo[0];
      }
    }
  }
}

// lse and loss of each row from its parts: 8 rows a block (32 bytes of each part), 32 threads a row.
__global__ void __launch_bounds__(kCeThreads)
ce_rows_kernel(const float2* __restrict__ stats, long long stats_ld, int parts, int rows, int V, const int32_t* __restrict__ labels,
               const float* __restrict__ target, float* __restrict__ lse, float* __restrict__ row_loss) {
  pdl_wait();
  pdl_launch_dependents();
  const int r = threadIdx.x & 7, y = threadIdx.x >> 3, row = blockIdx.x * 8 + r;
  float m = -INFINITY, s = 0.f;
  if (row < rows) {
#pragma unroll 4
    for (int i = y; i < parts; i += 32) {
      const float2 v = stats[(long long)i * stats_ld + row];
      if (v.y == 0.f) continue;              // a part without any class (its reference says nothing)
      const float top = fmaxf(m, v.x);
      if (top == INFINITY) { m = top; s = NAN; continue; }
      s = s * exp2f((m - top) * tc::kLog2e) + v.y * exp2f((v.x - top) * tc::kLog2e);
      m = top;
    }
  }
  __shared__ float ms[32][8], ss[32][8];
  ms[y][r] = m;
  ss[y][r] = s;
  __syncthreads();
  if (y || row >= rows) return;
  for (int i = 1; i < 32; ++i) m = fmaxf(m, ms[i][r]);
  float sum = 0.f;
  for (int i = 0; i < 32; ++i)
    if (ss[i][r] != 0.f) sum += ss[i][r] * exp2f((ms[i][r] - m) * tc::kLog2e);
  const float l = m + logf(sum);
  lse[row] = l;
  row_loss[row] = ce_counts(labels[row], V) ? l - target[row] : 0.f;
}

// Mean over the counted rows: one block, always in the same order.
__global__ void __launch_bounds__(kCeThreads)
ce_loss_kernel(const float* __restrict__ row_loss, int T, const CeHeader* __restrict__ hdr, float* __restrict__ loss) {
  pdl_wait();
  pdl_launch_dependents();
  double s = 0.0;
  for (int t = threadIdx.x; t < T; t += kCeThreads) s += (double)row_loss[t];
  __shared__ double part[kCeThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kCeThreads / 32; ++i) s += part[i];
    const int n = hdr->count;
    loss[0] = n > 0 ? (float)(s / n) : 0.f;
    loss[1] = (float)n;
  }
}

// Exponentials -> dl (without the factor g / count), in place, and the column sums of a slab of rows for dbias.
// A thread has 8 columns; `part_cols` columns share a reference in `stats`.
template <bool kF32>
__global__ void __launch_bounds__(kCeThreads)
ce_dl_kernel(__half* __restrict__ p, long long ld, long long plane, int rows, int V, int slab, const float2* __restrict__ stats,
             long long stats_ld, int part_cols, const float* __restrict__ lse, const float* __restrict__ target,
             const int32_t* __restrict__ labels, float* __restrict__ sums /* [slab][V] or null */) {
  pdl_wait();
  pdl_launch_dependents();
  const int col = (blockIdx.x * kCeThreads + threadIdx.x) * 8;
  if (col >= V) return;
  const float2* ref = stats + (long long)(col / part_cols) * stats_ld;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int r1 = min(rows, (int)(blockIdx.y + 1) * slab);
  for (int r = blockIdx.y * slab; r < r1; ++r) {
    const int label = labels[r];
    __half* q = p + (long long)r * ld + col;
    float v[8];
    if (ce_counts(label, V)) {
      const float f = exp2f(fmaf(ref[r].x - lse[r], tc::kLog2e, -tc::kCeExpBits));
      const uint4 h = *reinterpret_cast<const uint4*>(q);
      const uint32_t u[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) tc::half2_floats(u[i], v[2 * i], v[2 * i + 1]);
      if constexpr (kF32) {
        const uint4 l = *reinterpret_cast<const uint4*>(q + plane);
        const uint32_t w[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float a, b;
          tc::half2_floats(w[i], a, b);
          v[2 * i] += a;
          v[2 * i + 1] += b;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= f;
      if (label >= col && label < col + 8) {
        const float d = expm1f(target[r] - lse[r]);   // p - 1 without the cancellation
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j == label) v[j] = d;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += v[j];
    if constexpr (kF32) {
      __half hi[8], lo[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) tc::split_half(v[j] * kCeDlScale, hi[j], lo[j]);
      *reinterpret_cast<uint4*>(q) = make_uint4(tc::pack_half2(hi[0], hi[1]), tc::pack_half2(hi[2], hi[3]),
                                                tc::pack_half2(hi[4], hi[5]), tc::pack_half2(hi[6], hi[7]));
      *reinterpret_cast<uint4*>(q + plane) = make_uint4(tc::pack_half2(lo[0], lo[1]), tc::pack_half2(lo[2], lo[3]),
                                                        tc::pack_half2(lo[4], lo[5]), tc::pack_half2(lo[6], lo[7]));
    } else {
      *reinterpret_cast<uint4*>(q) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                                pack_bf16x2(v[6], v[7]));
    }
  }
  if (sums) {
    float* s = sums + (long long)blockIdx.y * V + col;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j < V) s[j] = acc[j];
  }
}

// dbias from the slabs' column sums.
__global__ void __launch_bounds__(kCeThreads)
ce_dbias_kernel(const float* __restrict__ sums, int slabs, int V, const CeHeader* __restrict__ hdr, void* __restrict__ dbias, int is_bf16) {
  pdl_wait();
  pdl_launch_dependents();
  const int v = blockIdx.x * kCeThreads + threadIdx.x;
  if (v >= V) return;
  float s = 0.f;
#pragma unroll 8
  for (int i = 0; i < slabs; ++i) s += sums[(long long)i * V + v];
  s *= hdr->grad_f;
  if (is_bf16) ((bf16*)dbias)[v] = __float2bfloat16_rn(s);
  else ((float*)dbias)[v] = s;
}

}  // namespace lp
