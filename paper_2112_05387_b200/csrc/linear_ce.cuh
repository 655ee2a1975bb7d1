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
  int done;           // blocks of the last pass over the rows that have finished
  int count;          // rows whose label is a class
  float logit_f;      // scale of x w^T's accumulator
  float dx_f, dw_f;   // scales of the gradients' accumulators
  float grad_f;       // g / count
  int dl_seen;        // pieces of the rows whose dl the product of dx has seen (see GemmParams)
};

__device__ __forceinline__ bool ce_counts(int label, int V) { return label >= 0 && label < V; }

// Number of rows that count, by one block; to thread 0.
__device__ __forceinline__ int ce_count_rows(const int32_t* labels, int T, int V) {
  int n = 0;
  for (int t0 = threadIdx.x; t0 < T; t0 += 8 * kCeThreads) {
    int label[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) label[k] = t0 + k * kCeThreads < T ? labels[t0 + k * kCeThreads] : -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) n += ce_counts(label[k], V);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
  __shared__ int cnt[kCeThreads / 32];
  if ((threadIdx.x & 31) == 0) cnt[threadIdx.x >> 5] = n;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 1; i < kCeThreads / 32; ++i) n += cnt[i];
  return n;
}

// fp32 problems: block 0 counts the rows, the others take the largest finite magnitudes of x and w (parts of each).  Rows of x that
// do not count and rows of w whose class is masked are left out: a large number in the padding would push the others out of the scaled
// parts' bits.
__global__ void __launch_bounds__(kCeThreads)
ce_prepare_kernel(const int32_t* __restrict__ labels, int T, int D, int V, const float* __restrict__ x, const float* __restrict__ w,
                  const float* __restrict__ bias, float* __restrict__ amax, int parts, CeHeader* __restrict__ hdr) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float part[kCeThreads / 32];
  if (blockIdx.x == 0) {
    const int n = ce_count_rows(labels, T, V);
    if (threadIdx.x == 0) {
      hdr->err = hdr->done = 0;
      hdr->count = n;
    }
    return;
  }
  const int b = blockIdx.x - 1;
  const bool of_w = b >= parts;
  const float* v = of_w ? w : x;
  const long long n = (long long)(of_w ? V : T) * D;
  const int k = of_w ? b - parts : b;
  const long long lo = n / 4 * k / parts, hi = n / 4 * (k + 1) / parts;
  float m = 0.f;
  auto take = [&](float a) {
    if (fabsf(a) <= 3.4028235e38f) m = fmaxf(m, fabsf(a));
  };
  auto row_of = [&](long long e, int cols) {   // (the division as in ce_pack_kernel)
    return n >> 32 ? e / cols : (long long)((uint32_t)e / (uint32_t)cols);
  };
  // (one load, whichever it is: a branch around it would stand between the reads of an unrolled loop)
  const int32_t* marks = of_w ? reinterpret_cast<const int32_t*>(bias) : labels;
  auto keep = [&](long long row) {
    const int32_t mark = __ldg(marks + row);
    return of_w ? __int_as_float(mark) != -INFINITY : ce_counts(mark, V);
  };
  const bool all = of_w && !bias;
  if (all || D % 4 == 0) {
    // (an access has elements of one row)
#pragma unroll 4
    for (long long i = lo + threadIdx.x; i < hi; i += kCeThreads) {
      float f[4];
      ldv(v + 4 * i, f);
      const bool take_it = all || keep(row_of(i, D / 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) take(take_it ? f[j] : 0.f);
    }
  } else {
#pragma unroll 2
    for (long long i = lo + threadIdx.x; i < hi; i += kCeThreads) {
      float f[4];
      ldv(v + 4 * i, f);
      long long r = row_of(4 * i, D);
      bool take_it = keep(r);
      int left = (int)((r + 1) * D - 4 * i);   // elements of the row from 4 i on
#pragma unroll
      for (int j = 0; j < 4; ++j, --left) {
        if (left == 0) {
          take_it = keep(++r);
          left = D;
        }
        take(take_it ? f[j] : 0.f);
      }
    }
  }
  if (k == 0 && threadIdx.x < n % 4) {
    const long long e = n - 1 - threadIdx.x;
    take(all || keep(row_of(e, D)) ? v[e] : 0.f);
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
// Rows of x whose label is no class become zeros: what stands there (padding, NaN) must not reach dw through a product with 0.  So do,
// in fp32 problems, the finite values of a masked class's row of w, which the scale does not know (its logit is -inf and its dl 0,
// whatever they are).
// Blocks [1, xb) take x, the rest w (none where it is used in place), block 0 nothing but the header (bf16 problems: the count of
// rows with it).  kVec: D is a multiple of 8.
template <bool kVec>
__global__ void __launch_bounds__(kCeThreads)
ce_pack_kernel(const void* __restrict__ x, const void* __restrict__ w, const void* __restrict__ bias, const int32_t* __restrict__ labels, int is_bf16,
               int T, int D, int V, long long ld, __half* __restrict__ xo, long long x_plane, __half* __restrict__ wo, long long w_plane, int xb,
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
  if (blockIdx.x == 0) {
    const int counted = is_bf16 ? ce_count_rows(labels, T, V) : hdr->count;
    if (threadIdx.x) return;
    if (is_bf16) {
      hdr->err = hdr->done = 0;
      hdr->count = counted;
    }
    hdr->dl_seen = 0;
    const float gf = counted > 0 ? g / (float)counted : 0.f;
    const float dl = is_bf16 ? 1.f : 1.f / kCeDlScale;
    hdr->logit_f = (1.f / scales[0]) * (1.f / scales[1]);
    hdr->grad_f = gf;
    hdr->dx_f = gf * dl * (1.f / scales[1]);
    hdr->dw_f = gf * dl * (1.f / scales[0]);
    return;
  }
  const bool of_w = (int)blockIdx.x >= xb;
  const int blk = of_w ? blockIdx.x - xb : blockIdx.x - 1, blks = of_w ? gridDim.x - xb : xb - 1;
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
    const bool masked = of_w && !is_bf16 && bias && ((const float*)bias)[r] == -INFINITY;
    auto scaled = [&](float a) { return !keep || (masked && fabsf(a) <= 3.4028235e38f) ? 0.f : a * scale; };
    if (is_bf16) {
      if constexpr (kVec) {
        uint4 v = ld_raw((const bf16*)src + from);
        if (!keep) v = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>((bf16*)dst + at) = v;
      } else {
        ((bf16*)dst)[at] = keep ? ((const bf16*)src)[from] : __float2bfloat16_rn(0.f);
      }
    } else {
      if constexpr (kVec) {
        float v[4], z[4];
        uint32_t hi[4], lo[4];
        ldv((const float*)src + from, v);
        ldv((const float*)src + from + 4, z);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          tc::split_f16x2(scaled(v[2 * j]), scaled(v[2 * j + 1]), hi[j], lo[j]);
          tc::split_f16x2(scaled(z[2 * j]), scaled(z[2 * j + 1]), hi[2 + j], lo[2 + j]);
        }
        *reinterpret_cast<uint4*>(dst + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(dst + plane + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      } else {
        __half hi, lo;
        tc::split_half(scaled(((const float*)src)[from]), hi, lo);
        dst[at] = hi;
        dst[plane + at] = lo;
      }
    }
  }
}

// Joins a part (maximum, sum of exponentials relative to it) to another.  A part without any class has the sum 0, and its
// reference says nothing; an infinite logit makes the sum NaN, as inf - inf is.
__device__ __forceinline__ void ce_join(float& m, float& s, const float2 v) {
  if (v.y == 0.f) return;
  if (s == 0.f) {
    m = v.x;
    s = v.x == INFINITY ? NAN : v.y;
    return;
  }
  const float top = fmaxf(m, v.x);
  s = s * exp2f((m - top) * tc::kLog2e) + v.y * exp2f((v.x - top) * tc::kLog2e);
  m = top;
}

// Every 32nd part of a row from `first` on, kBatch reads on their way together (left to the compiler they go one by one, 2011 rows of
// 391 parts 18 us) and one maximum for all of them.
template <int kBatch>
__device__ __forceinline__ void ce_join_parts(float& m, float& s, const float2* stats, long long ld, int first, int parts) {
#pragma unroll 1
  for (int i = first; i < parts; i += 32 * kBatch) {
    float2 v[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) v[k] = i + 32 * k < parts ? stats[(i + 32 * k) * ld] : make_float2(0.f, 0.f);
    float top = m;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = v[k].y == 0.f ? top : fmaxf(top, v[k].x);
    if (s != 0.f) s *= exp2f((m - top) * tc::kLog2e);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) s += v[k].y == 0.f ? 0.f : v[k].y * exp2f((v[k].x - top) * tc::kLog2e);
    m = top;
  }
}

// The joined parts of a warp's lanes, to all of them.  (Both lanes of an exchange add the same two terms, the lower lane's first:
// the same bits.)
__device__ __forceinline__ void ce_join_warp(float& m, float& s) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float2 v = make_float2(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
    float a = lane & o ? v.x : m, b = lane & o ? v.y : s;
    ce_join(a, b, lane & o ? make_float2(m, s) : v);
    m = a;
    s = b;
  }
}

// Loss of a row from its maximum and the sum of exponentials relative to it.  lse stays in these two parts, for the gradients `top` and,
// in the place of the label's logit, the logarithm: where that logit is the maximum, the loss is the logarithm alone, and a rounding
// of lse itself (2^-24 of logits that may be large) would be most of a small loss and of its gradients.
__device__ __forceinline__ float ce_row_loss(float m, float log_sum, float target) { return (m - target) + log_sum; }

// Loss of each row from its parts, and what the gradients need of lse: 8 rows a block (64 bytes of each part), 32 threads a row.  On the last piece of the
// rows (`loss` given) the block that finishes last takes the mean over the counted rows of all T, in the order of the rows.
__global__ void __launch_bounds__(kCeThreads)
ce_rows_kernel(const float2* __restrict__ stats, long long stats_ld, int parts, int r0, int rows, int T, int V,
               const int32_t* __restrict__ labels, float* __restrict__ target, float* __restrict__ top, float* __restrict__ row_loss,
               CeHeader* __restrict__ hdr, float* __restrict__ loss) {
  pdl_wait();
  pdl_launch_dependents();
  const int r = threadIdx.x & 7, y = threadIdx.x >> 3, row = blockIdx.x * 8 + r;
  float m = -INFINITY, s = 0.f;
  if (row < rows) {
    ce_join_parts<8>(m, s, stats + row, stats_ld, y, parts);
  }
  __shared__ float ms[8][33], ss[8][33];
  ms[r][y] = m;
  ss[r][y] = s;
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = blockIdx.x * 8 + warp;   // a warp joins the parts of a row
  m = ms[warp][lane];
  s = ss[warp][lane];
  ce_join_warp(m, s);
  if (lane == 0 && t < rows) {
    const float l = logf(s);
    row_loss[r0 + t] = ce_counts(labels[r0 + t], V) ? ce_row_loss(m, l, target[r0 + t]) : 0.f;
    top[r0 + t] = m;
    target[r0 + t] = l;
    __threadfence();
  }
  if (!loss) return;
  __syncthreads();
  __shared__ int last;
  if (threadIdx.x == 0) last = atomicAdd(&hdr->done, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  double sum = 0.0;
  for (int t0 = threadIdx.x; t0 < T; t0 += 8 * kCeThreads) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = t0 + k * kCeThreads < T ? __ldcg(row_loss + t0 + k * kCeThreads) : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += (double)v[k];
  }
  __shared__ double part[kCeThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  const int n = ce_count_rows(labels, T, V);   // (its barrier is that of `part`, too)
  if (threadIdx.x == 0) {
    for (int i = 1; i < kCeThreads / 32; ++i) sum += part[i];
    loss[0] = n > 0 ? (float)(sum / n) : 0.f;
    loss[1] = (float)n;
  }
}

// All of it at once for few rows and parts, in one block: the loss of each row, a warp each, the number of counted rows and
// the mean.
__global__ void __launch_bounds__(1024)
ce_finish_kernel(const float2* __restrict__ stats, long long stats_ld, int parts, int rows, int V, const int32_t* __restrict__ labels,
                 float* __restrict__ target, float* __restrict__ top, float* __restrict__ row_loss, float* __restrict__ loss) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  double total = 0.0;
  int count = 0;
  for (int row = warp; row < rows; row += 32) {
    // (read ahead of the parts)
    const bool counts = ce_counts(labels[row], V);
    const float logit = target[row];
    float m = -INFINITY, s = 0.f;
    ce_join_parts<4>(m, s, stats + row, stats_ld, lane, parts);
    ce_join_warp(m, s);
    const float l = logf(s), x = counts ? ce_row_loss(m, l, logit) : 0.f;
    if (lane == 0) {
      row_loss[row] = x;
      top[row] = m;
      target[row] = l;
    }
    total += (double)x;
    count += counts;
  }
  __shared__ double totals[32];
  __shared__ int counts_s[32];
  if (lane == 0) {
    totals[warp] = total;
    counts_s[warp] = count;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 32; ++w) {
      total += totals[w];
      count += counts_s[w];
    }
    loss[0] = count > 0 ? (float)(total / count) : 0.f;
    loss[1] = (float)count;
  }
}

// Loss alone of at most four rows: a pass over w that its bytes bound (a tile of the tensor cores holds 128 rows, and fetches w
// in rows of 128 bytes: 105 us for one row, 2048 x 100000 in bf16, 64 us of bytes).  A warp has four classes at a time, each lane 16 bytes of each of
// them a step; x stands in shared memory in fp32.  Every block joins its warps' maxima and sums to one part.
template <typename T, int kRows, bool kVec>
__global__ void __launch_bounds__(kCeThreads)
ce_few_kernel(const T* __restrict__ x, const T* __restrict__ w, const T* __restrict__ bias, const int32_t* __restrict__ labels, int rows, int D,
              int V, float2* __restrict__ stats, long long stats_ld, float* __restrict__ target, CeHeader* __restrict__ hdr) {
  extern __shared__ __align__(16) float few_x[];   // [kRows][D]
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) hdr->err = 0;
  for (int i = threadIdx.x; i < kRows * D; i += kCeThreads) few_x[i] = i < rows * D ? to_f(x[i]) : 0.f;
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int N = kVec ? VecT<T>::N : 1;
  float m[kRows], s[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) { m[r] = -INFINITY; s[r] = 0.f; }
  for (int v0 = (blockIdx.x * 8 + warp) * 4; v0 < V; v0 += gridDim.x * 32) {
    const T* at[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) at[c] = w + (long long)min(v0 + c, V - 1) * D;
    float acc[4][kRows] = {};
#pragma unroll 2
    for (int d = lane * N; d < D; d += 32 * N) {
      float f[4][N];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if constexpr (kVec) ldv(at[c] + d, f[c]);
        else f[c][0] = to_f(at[c][d]);
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float xv = few_x[r * D + d + j];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c][r] = fmaf(f[c][j], xv, acc[c][r]);
        }
    }
    float b[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) b[c] = v0 + c < V ? (bias ? to_f(bias[v0 + c]) : 0.f) : -INFINITY;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      float l[4], top = m[r];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        l[c] = warp_sum(acc[c][r]);
        l[c] = v0 + c < V ? l[c] + b[c] : -INFINITY;
        if (r < rows && lane == 0 && labels[r] == v0 + c) target[r] = l[c];
        top = fmaxf(top, l[c]);
      }
      if (top == -INFINITY && l[0] == l[0] && l[1] == l[1] && l[2] == l[2] && l[3] == l[3]) continue;   // (no class yet, and no NaN)
      float sum = s[r] == 0.f ? 0.f : s[r] * exp2f((m[r] - top) * tc::kLog2e);
#pragma unroll
      for (int c = 0; c < 4; ++c) sum += exp2f((l[c] - top) * tc::kLog2e);
      s[r] = sum;
      m[r] = top;
    }
  }
  __shared__ float2 parts[8][kRows];
  if (lane == 0)
#pragma unroll
    for (int r = 0; r < kRows; ++r) parts[warp][r] = make_float2(m[r], s[r]);
  __syncthreads();
  if (threadIdx.x < rows) {
    float a = -INFINITY, b = 0.f;
    for (int i = 0; i < 8; ++i) ce_join(a, b, parts[i][threadIdx.x]);
    stats[(long long)blockIdx.x * stats_ld + threadIdx.x] = make_float2(a, b);
  }
}

// Exponentials -> dl (without the factor g / count), in place, and the column sums of a slab of rows for dbias: the block's slab in
// `sums`, or dbias itself where one slab is all there is.  A warp has 256 columns of every eighth row, a thread 8 of them;
// `part_cols` columns share a reference in `stats`.
// Rows are taken a few at a time, all their reads ahead of the first write (348 x 3000: 12.3 -> 10.1 us).  Many rows are bound by
// HBM, read and written in place: 4096 x 32000 114 us, 4.6 TB/s (blocks of 512, 1024 or 2048 columns 112 to 118; the rows that the
// product wrote last first 132).
constexpr int kCeSlab = 64;
template <bool kF32>
__global__ void __launch_bounds__(kCeThreads)
ce_dl_kernel(__half* __restrict__ p, long long ld, long long plane, int rows, int V, const float2* __restrict__ stats, long long stats_ld,
             int part_cols, const float* __restrict__ top, const float* __restrict__ log_sum, const float* __restrict__ row_loss,
             const int32_t* __restrict__ labels, float* __restrict__ sums /* [slab][V] or null */, void* __restrict__ dbias /* or null */, const CeHeader* __restrict__ hdr) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = blockIdx.x * 256 + lane * 8;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (col < V) {
    const float2* ref = stats + (long long)(col / part_cols) * stats_ld;
    const int r1 = min(rows, (int)(blockIdx.y + 1) * kCeSlab);
    constexpr int kBatch = kF32 ? 2 : 4;   // rows whose exponentials are on their way together
    for (int r0 = blockIdx.y * kCeSlab + warp; r0 < r1; r0 += 8 * kBatch) {
      uint4 hs[kBatch], ls[kF32 ? kBatch : 1];
      int labels_r[kBatch];
      float tops[kBatch], logs[kBatch], refs[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int r = min(r0 + 8 * k, r1 - 1);
        hs[k] = *reinterpret_cast<const uint4*>(p + (long long)r * ld + col);
        if constexpr (kF32) ls[k] = *reinterpret_cast<const uint4*>(p + plane + (long long)r * ld + col);
        labels_r[k] = labels[r];
        tops[k] = top[r];
        logs[k] = log_sum[r];
        refs[k] = ref[r].x;
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int r = r0 + 8 * k, label = labels_r[k];
        if (r >= r1) break;
        __half* q = p + (long long)r * ld + col;
        float v[8];
        if (ce_counts(label, V)) {
          const float f = exp2f(fmaf((refs[k] - tops[k]) - logs[k], tc::kLog2e, -tc::kCeExpBits));
          const uint32_t u[4] = {hs[k].x, hs[k].y, hs[k].z, hs[k].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) tc::half2_floats(u[i], v[2 * i], v[2 * i + 1]);
          if constexpr (kF32) {
            const uint32_t w[4] = {ls[k].x, ls[k].y, ls[k].z, ls[k].w};
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
            const float d = expm1f(-row_loss[r]);   // p - 1 without the cancellation
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
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) tc::split_f16x2(v[2 * j] * kCeDlScale, v[2 * j + 1] * kCeDlScale, hi[j], lo[j]);
          *reinterpret_cast<uint4*>(q) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(q + plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        } else {
          *reinterpret_cast<uint4*>(q) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                                    pack_bf16x2(v[6], v[7]));
        }
      }
    }
  }
  if (!sums && !dbias) return;
  __shared__ float part[8][256];
#pragma unroll
  for (int j = 0; j < 8; ++j) part[warp][lane * 8 + j] = acc[j];
  __syncthreads();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= V) return;
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += part[w][threadIdx.x];
  if (sums) sums[(long long)blockIdx.y * V + c] = s;
  else if (kF32) ((float*)dbias)[c] = s * hdr->grad_f;
  else ((bf16*)dbias)[c] = __float2bfloat16_rn(s * hdr->grad_f);
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
