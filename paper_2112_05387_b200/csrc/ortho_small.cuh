// Orthogonalisation of small matrices in one launch: everything of a matrix stays in shared memory.
//
// With 15 dependent products of a few tiles each, a small matrix is bound by launches and by the way through global memory
// and back (16 x 144: 85 us, its bytes take 10 ns).  Here a cluster of C CTAs holds X (smaller side S <= 128 padded to 16, 32, 64
// or 128; the larger side in C slices) as fp16 high and low parts from the first pass to the last:
//   partial = X_slice X_slice^T in every CTA;  cluster barrier;  every CTA adds up its share of the C partials and writes it to
//   all (distributed shared memory);  cluster barrier;  B = a I + b A + c A^2 in every CTA;  X_slice <- B X_slice in place.
// Products are warp-level (mma.sync m16n8k16): the operands change hands between warps every few hundred cycles, and nothing is
// large enough for the tensor memory's 128 rows to pay.  Sums of more than two K steps are added up in fp32 registers.
#pragma once
#include <cuda_fp16.h>

#include "ortho.cuh"

namespace lp {

constexpr int kSmallThreads = 256;
constexpr int kSmallWarps = kSmallThreads / 32;

struct OrthoSmall {
  OrthoSource src;
  int s, l;               // smaller and larger side
  int tall;               // the matrix is l x s in memory
  int slice, ctas;        // columns of a CTA's slice (a multiple of 16), CTAs of a cluster
  int steps;
  float a, b, c, eps;
  void* out;
  int out_bf16, update;
  float keep, step;
  int* err;               // cleared, or null
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], const __half* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(tc::smem_u32(p)) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], const __half* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(tc::smem_u32(p)) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_b32x2(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}

// Shared memory: planes of X [2][S][slice + 8], of A [P][S][S + 8], then the partial sums [G][S][S] fp32 and, in the same place
// later, the planes of B [P][S][S + 8].  P: 2 for fp32 results, else 1 (A and B are fp16).  The warps share X X^T as tiles of 16
// rows and small_cols() columns, G groups of them K where there are fewer tiles than warps.
__host__ __device__ constexpr int small_cols(int S) { return S == 16 ? 16 : (S == 128 ? 64 : 32); }
__host__ __device__ constexpr int small_groups(int S) { return S == 16 ? 8 : (S == 32 ? 4 : 1); }
__host__ __device__ inline size_t small_smem(int S, int slice, bool split) {
  const size_t mat = (size_t)(split ? 2 : 1) * S * (S + 8) * 2, part = (size_t)small_groups(S) * S * S * 4;
  return (size_t)2 * S * (slice + 8) * 2 + mat + (mat > part ? mat : part);
}

// Products of the 16 x 16 NB tile (m0, n0) of P Q^T over K columns [k0, k1): planes of P and Q `pl` elements apart, rows `ld`.
// kSplit: all parts but lo * lo.
template <bool kSplit, int NB>
__device__ __forceinline__ void small_tile(float (&sum)[NB][2][4], const __half* P, const __half* Q, int pl, int ld, int m0, int n0, int k0,
                                           int k1, int lane) {
  const __half* pa = P + (m0 + (lane & 15)) * ld + (lane >> 4) * 8;
  // two 8-row tiles of Q: lanes 0-7 rows n0.., 8-15 the same 8 columns on, 16-31 rows n0 + 8..
  const __half* qb = Q + (n0 + (lane & 7) + ((lane >> 4) << 3)) * ld + ((lane >> 3) & 1) * 8;
#pragma unroll 1
  for (int k = k0; k < k1; k += 32) {
    float acc[NB][2][4] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kk = k + 16 * h;
      if (kk >= k1) break;
      uint32_t ah[4], al[4], bh[NB][4], bl[NB][4];
      ldsm4(ah, pa + kk);
      if constexpr (kSplit) ldsm4(al, pa + pl + kk);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        ldsm4(bh[n], qb + 16 * n * ld + kk);
        if constexpr (kSplit) ldsm4(bl[n], qb + pl + 16 * n * ld + kk);
      }
      if constexpr (kSplit) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int t = 0; t < 2; ++t) mma_f16(acc[n][t], ah, bl[n][2 * t], bl[n][2 * t + 1]);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int t = 0; t < 2; ++t) mma_f16(acc[n][t], al, bh[n][2 * t], bh[n][2 * t + 1]);
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) mma_f16(acc[n][t], ah, bh[n][2 * t], bh[n][2 * t + 1]);
    }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[n][t][i] += acc[n][t][i];
  }
}

template <bool kSplit, int S>
__global__ void __launch_bounds__(kSmallThreads, S <= 64 ? 2 : 1)
ortho_small_kernel(const __grid_constant__ OrthoSmall q) {
  extern __shared__ __align__(16) uint8_t small_smem_raw[];
  constexpr int P = kSplit ? 2 : 1, G = small_groups(S), LD = S + 8;
  constexpr float kX = 4096.f, kA = 1024.f, kB = 1024.f;   // as in ortho_run
  const int ldx = q.slice + 8, xpl = S * ldx;
  __half* X = reinterpret_cast<__half*>(small_smem_raw);
  __half* A = X + 2 * xpl;
  float* part = reinterpret_cast<float*>(A + P * S * LD);
  __half* B = reinterpret_cast<__half*>(part);
  __shared__ double sums[kSmallWarps];
  __shared__ double cta_sum;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();
  const int mat = blockIdx.x / q.ctas;
  const long long base = q.src.use_off ? q.src.off[mat] : mat * q.src.elems;
  const int j0 = (int)rank * q.slice, width = max(0, min(q.slice, q.l - j0));   // this CTA's columns

  pdl_wait();
  pdl_launch_dependents();
  if (q.err && blockIdx.x == 0 && threadIdx.x == 0) *q.err = 0;

  // element e of the slice: row i of X, column j0 + j; contiguous in memory along j (wide) or i (tall)
  const int n = q.s * width, inner = q.tall ? q.s : max(width, 1);
  auto place = [&](int e, int& i, int& j, long long& at) {
    const int hi = (int)((uint32_t)e / (uint32_t)inner), lo = e - hi * inner;
    i = q.tall ? lo : hi;
    j = q.tall ? hi : lo;
    at = base + (q.tall ? (long long)(j0 + j) * q.s + i : (long long)i * q.l + j0 + j);
  };
  double sum = 0.0;
#pragma unroll 4
  for (int e = threadIdx.x; e < n; e += kSmallThreads) {
    int i, j;
    long long at;
    place(e, i, j, at);
    float u[1], m[1];
    ortho_load<false>(q.src.g, q.src.g_bf16, at, u);
    if (q.src.momentum) {
      m[0] = fmaf(q.src.mu, q.src.momentum[at], u[0]);
      q.src.momentum[at] = m[0];
      ortho_direction(q.src, u, m);
    }
    sum += (double)u[0] * (double)u[0];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sums[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSmallWarps; ++w) sum += sums[w];
    cta_sum = sum;
  }
  // (rows and columns of the padding are zeros, and stay zeros)
  for (int e = threadIdx.x; e < 2 * xpl / 8; e += kSmallThreads) reinterpret_cast<uint4*>(X)[e] = make_uint4(0u, 0u, 0u, 0u);
  __syncthreads();
  tc::cluster_sync_all();
  sum = 0.0;
  for (int r = 0; r < q.ctas; ++r) sum += ld_cluster_f64(tc::mapa_u32(tc::smem_u32(&cta_sum), r));
  const float scale = (float)((double)kX / fmax(sqrt(sum), (double)q.eps));
#pragma unroll 4
  for (int e = threadIdx.x; e < n; e += kSmallThreads) {
    int i, j;
    long long at;
    place(e, i, j, at);
    float u[1], m[1];
    ortho_load<false>(q.src.g, q.src.g_bf16, at, u);
    if (q.src.momentum) {
      m[0] = q.src.momentum[at];
      ortho_direction(q.src, u, m);
    }
    __half hi, lo;
    tc::split_half(u[0] * scale, hi, lo);
    X[i * ldx + j] = hi;
    X[xpl + i * ldx + j] = lo;
  }
  __syncthreads();

  const int g = lane >> 2, t2 = 2 * (lane & 3);   // accumulator fragment: rows g, g + 8, columns t2, t2 + 1
  constexpr int kCols = small_cols(S), NB = kCols / 16, kAcross = S / kCols, kTiles = S / 16 * kAcross;
  constexpr int kMine = (kTiles + kSmallWarps - 1) / kSmallWarps;     // of a warp, where no group shares K
  static_assert(kTiles * G % kSmallWarps == 0 || kTiles * G < kSmallWarps, "tiles over the warps");
  for (int step = 0; step < q.steps; ++step) {
    const bool last = step + 1 == q.steps;
    // partial sums of X X^T
#pragma unroll 1
    for (int w = warp; w < kTiles * G; w += kSmallWarps) {
      const int tile = w % kTiles, grp = w / kTiles;
      const int m0 = tile / kAcross * 16, n0 = tile % kAcross * kCols, ks = q.slice / 16;
      float acc[NB][2][4] = {};
      small_tile<kSplit, NB>(acc, X, X, xpl, ldx, m0, n0, ks * grp / G * 16, ks * (grp + 1) / G * 16, lane);
      float* o = part + grp * S * S + (m0 + g) * S + n0 + t2;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          *reinterpret_cast<float2*>(o + 16 * n + 8 * t) = make_float2(acc[n][t][0], acc[n][t][1]);
          *reinterpret_cast<float2*>(o + 8 * S + 16 * n + 8 * t) = make_float2(acc[n][t][2], acc[n][t][3]);
        }
    }
    __syncwarp();
    tc::cluster_sync_all();
    // each CTA adds up its share of the entries (the same order whatever the CTA), four a thread with all CTAs' sums on their way
    // before the first is added, and writes them into every CTA's A: an entry crosses between SMs C times, not C^2
    const int share = S * S / q.ctas;
    for (int e = (int)rank * share + threadIdx.x * 4; e < (int)(rank + 1) * share; e += kSmallThreads * 4) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < G; ++k) {
        float4 x[8];
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r < q.ctas) x[r] = tc::ld_cluster_f32x4(tc::mapa_u32(tc::smem_u32(part + k * S * S + e), r));
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r < q.ctas) { v[0] += x[r].x; v[1] += x[r].y; v[2] += x[r].z; v[3] += x[r].w; }
      }
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) tc::split_f16x2(v[2 * i] * (kA / (kX * kX)), v[2 * i + 1] * (kA / (kX * kX)), hi[i], lo[i]);
      const uint32_t at = tc::smem_u32(A + e / S * LD + e % S);
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < q.ctas) {
          const uint32_t to = tc::mapa_u32(at, r);
          st_cluster_b32x2(to, hi[0], hi[1]);
          if constexpr (kSplit) st_cluster_b32x2(to + S * LD * 2, lo[0], lo[1]);
        }
    }
    __syncwarp();
    tc::cluster_sync_all();   // A is complete everywhere, and the partial sums have been read: B may take their place
#pragma unroll
    for (int u = 0; u < kMine; ++u) {
      const int tile = warp + u * kSmallWarps;
      if (tile >= kTiles) break;
      const int m0 = tile / kAcross * 16, n0 = tile % kAcross * kCols;
      float bv[NB][2][4] = {};
      small_tile<kSplit, NB>(bv, A, A, S * LD, LD, m0, n0, 0, S, lane);
      const float fa = q.b * (kB / kA), fc = q.c * (kB / (kA * kA));
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = m0 + g + 8 * h, c = n0 + 16 * n + 8 * t + t2, at = r * LD + c;
            float a0, a1;
            tc::half2_floats(*reinterpret_cast<const uint32_t*>(A + at), a0, a1);
            if constexpr (kSplit) {
              float l0, l1;
              tc::half2_floats(*reinterpret_cast<const uint32_t*>(A + S * LD + at), l0, l1);
              a0 += l0;
              a1 += l1;
            }
            uint32_t hi, lo;
            tc::split_f16x2(fmaf(fc, bv[n][t][2 * h], fa * a0) + (r == c ? q.a * kB : 0.f),
                            fmaf(fc, bv[n][t][2 * h + 1], fa * a1) + (r == c + 1 ? q.a * kB : 0.f), hi, lo);
            *reinterpret_cast<uint32_t*>(B + at) = hi;
            if constexpr (kSplit) *reinterpret_cast<uint32_t*>(B + S * LD + at) = lo;
          }
    }
    __syncthreads();
    // X <- B X in place: a warp has 16 rows (their part of B stays in its registers) of a strip of 16 columns, the warps together
    // all rows of 8 / (S / 16) strips a pass.  Everything of a strip is in registers before any of it is written.
    constexpr int kK = S / 16, kStrips = kSmallWarps / kK;
    const int m0 = warp % kK * 16;
    uint32_t bh[kK][4], bl[kSplit ? kK : 1][4];
#pragma unroll
    for (int k = 0; k < kK; ++k) {
      const __half* from = B + (m0 + (lane & 15)) * LD + 16 * k + (lane >> 4) * 8;
      ldsm4(bh[k], from);
      if constexpr (kSplit) ldsm4(bl[k], from + S * LD);
    }
#pragma unroll 1
    for (int s0 = 0; s0 < q.slice / 16; s0 += kStrips) {
      const int n0 = (s0 + warp / kK) * 16;
      const bool mine = n0 < q.slice;
      float lo_acc[2][4] = {}, hi_acc[2][4] = {};
      if (mine) {
        // lanes 0-7 rows k.. of 8 columns, 8-15 the next 8 rows, 16-31 the same of the next 8 columns
        const __half* from = X + (lane & 15) * ldx + n0 + (lane >> 4) * 8;
#pragma unroll
        for (int k = 0; k < kK; ++k) {
          uint32_t xh[4], xl[4];
          ldsm4_trans(xh, from + 16 * k * ldx);
          ldsm4_trans(xl, from + xpl + 16 * k * ldx);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            mma_f16(lo_acc[t], bh[k], xl[2 * t], xl[2 * t + 1]);
            if constexpr (kSplit) mma_f16(lo_acc[t], bl[k], xh[2 * t], xh[2 * t + 1]);
            mma_f16(hi_acc[t], bh[k], xh[2 * t], xh[2 * t + 1]);
          }
        }
      }
      __syncthreads();
      if (!mine) continue;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int i = m0 + g + 8 * h, j = n0 + 8 * t + t2;
          const float v[2] = {(hi_acc[t][2 * h] + lo_acc[t][2 * h]) * (1.f / kB), (hi_acc[t][2 * h + 1] + lo_acc[t][2 * h + 1]) * (1.f / kB)};
          if (!last) {
            uint32_t hi, lo;
            tc::split_f16x2(v[0], v[1], hi, lo);
            *reinterpret_cast<uint32_t*>(X + i * ldx + j) = hi;
            *reinterpret_cast<uint32_t*>(X + xpl + i * ldx + j) = lo;
          } else if (i < q.s) {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              if (j + d >= width) continue;
              const long long at = base + (q.tall ? (long long)(j0 + j + d) * q.s + i : (long long)i * q.l + j0 + j + d);
              float x = v[d] * (1.f / kX);
              if (q.out_bf16) {
                bf16* o = (bf16*)q.out + at;
                if (q.update) x = fmaf(q.step, x, q.keep * __bfloat162float(*o));
                *o = __float2bfloat16_rn(x);
              } else {
                float* o = (float*)q.out + at;
                if (q.update) x = fmaf(q.step, x, q.keep * *o);
                *o = x;
              }
            }
          }
        }
    }
    __syncthreads();
  }
  tc::cluster_sync_all();   // no CTA leaves while another may read its partial sums
}

}  // namespace lp
