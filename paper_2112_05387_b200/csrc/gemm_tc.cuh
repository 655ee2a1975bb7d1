// Dense batched matrix products on the tensor cores for the operators at the end of a training step (linear_ce.cuh,
// ortho.cuh): D[b] = A[b] B[b]^T with 16-bit operands and fp32 accumulation, each operand stored with either dimension
// contiguous, and the operator's own arithmetic in the epilogue.
//
// Tiles.  A CTA pair (cta_group::2) computes 256 x 256: each CTA holds 128 rows of A and 128 of B's 256 rows, and every
// tcgen05.mma reads both halves, so a 64-wide K block costs an SM 32 KB of loads for 128 x 256 x 64 products -- 64 bytes a
// cycle, what an SM draws from L2.  Products with too few such tiles to fill the SMs take 128 x 128 tiles on single CTAs.
// The grid is persistent: a CTA (pair) walks the tiles, six stages of operands in flight, two accumulators in tensor
// memory, so that a tile's epilogue runs under the next tile's products.
//
// Precision.  A product may be a sum of several: operands kept as a 16-bit high and a low part (planes of the same
// tensor) are multiplied as hi*hi + hi*lo + lo*hi in one accumulation (`nseg`, planes per segment).  Where fp32 results are
// wanted (kRounds), the tensor core's accumulator is emptied every `round_len` K blocks into registers and added up there:
// the accumulation inside the tensor core does not round to nearest, and its error grows with the number of K steps.
//
// Roles (320 threads): warp 0 TMA producer, warp 1 MMA issuer (of the pair's leader), warps 2..9 epilogue: two warps per
// quarter of the accumulator's rows, each taking one half of its columns; a thread has one row.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace lp {
namespace tc {

constexpr int kGemmStages = 6;
constexpr int kGemmThreads = 320;
constexpr int kGemmEpiWarps = 8;
constexpr uint32_t kGemmStageBytes = 32768;   // 128 rows x 64 columns of A and of B, 16 bits each
constexpr int kGemmScratchFloats = 32 * 33;   // per epilogue warp: a 32 x 32 block, to be written row by row
constexpr int kGemmMaxOffsets = 64;

struct GemmTail {
  uint64_t full[kGemmStages], empty[kGemmStages];
  uint64_t tmem_full[2], tmem_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};
constexpr size_t kGemmSmem = 1024 + (size_t)kGemmStages * kGemmStageBytes + (size_t)kGemmEpiWarps * kGemmScratchFloats * 4 + sizeof(GemmTail);
static_assert(kGemmSmem <= 232448, "shared memory of a block");

enum GemmEpi {
  EPI_H16 = 0,   // 16-bit planes of an intermediate: fp16 high (and low) part of f * acc (+ b * aux + diag)
  EPI_OUT = 1,   // a result in the caller's type: f * acc (+ what earlier pieces added up), or an update of weights with it
  EPI_CE = 2,    // logits: per row and column half the maximum, the sum of exponentials and the exponentials themselves
};

struct GemmParams {
  int M, N, batch;
  int tiles_m, tiles_n, total_tiles;
  int sym;                        // D is symmetric: tiles on and above the diagonal, written to both places (M = N)
  int group_m;                    // row tiles that are walked together (they share B tiles in L2)
  int kblocks, nseg;
  int a_z[3], b_z[3];             // first plane of each segment's operands
  int round_len;                  // kRounds: (K block, segment) steps per accumulation
  int a_mn, b_mn;                 // 1: the operand's row index is the contiguous one
  uint32_t idesc;
  int* err;
  // scale of the accumulator: f * f_dev[b]^f_pow
  float f;
  const float* f_dev;
  int f_pow;
  // EPI_H16
  __half* h_out;
  long long h_ld, h_batch, h_plane;   // elements; h_plane 0: no low part
  const __half* aux;                  // same geometry as h_out
  float aux_f, diag;
  // EPI_OUT
  void* out;
  int out_bf16;
  long long out_ld, out_batch;
  float* acc;                     // fp32 sums over pieces, [M][N], or null
  int acc_first, acc_last;        // first piece: stored, not added; last piece: the result goes to `out`
  // update of weights: out <- keep * out + step * value
  int update;
  float keep, step;
  int use_off;
  long long off[kGemmMaxOffsets]; // use_off: element offset of matrix b from `out`
  // EPI_CE
  const void* bias;               // [N] in the operands' type or null
  int bias_bf16;
  const int32_t* labels;          // [M]
  float2* stats;                  // [column half][M]: maximum, sum of exponentials
  long long stats_ld;
  float* target;                  // [M]: the label's logit
  // (h_out, h_ld, h_plane: exponentials relative to the half's maximum, times 2^14; null: not kept)
};

// Tile t of the walk -> batch, row tile, column tile.
__device__ __forceinline__ void gemm_tile(const GemmParams& p, int t, int& b, int& tm, int& tn) {
  if (p.sym) {
    const int per = p.tiles_m * (p.tiles_m + 1) / 2;
    b = t / per;
    int r = t - b * per;
    tm = 0;
    while (r >= p.tiles_m - tm) { r -= p.tiles_m - tm; ++tm; }
    tn = tm + r;
    return;
  }
  const int per = p.tiles_m * p.tiles_n;
  b = t / per;
  const int r = t - b * per;
  const int span = p.group_m * p.tiles_n;
  const int g = r / span, in = r - g * span;
  const int rows = min(p.group_m, p.tiles_m - g * p.group_m);
  tn = in / rows;
  tm = g * p.group_m + in - tn * rows;
}

__device__ __forceinline__ float gemm_scale(const GemmParams& p, int b) {
  float f = p.f;
  if (p.f_pow) {
    const float d = p.f_dev[b];
    f *= d;
    if (p.f_pow == 2) f *= d;
  }
  return f;
}

// fp16 high and low part of v: together 22 bits (the low part is rounded once).
__device__ __forceinline__ void split_half(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}
__device__ __forceinline__ uint32_t pack_half2(__half a, __half b) {
  return (uint32_t)__half_as_ushort(a) | ((uint32_t)__half_as_ushort(b) << 16);
}
__device__ __forceinline__ void half2_floats(uint32_t u, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
  a = f.x;
  b = f.y;
}

// One 32-column group of EPI_H16.  `row` < M; columns from `col` on; the group may run past N (the buffer's rows are
// padded to whole groups of 32 columns, and what lies there is never read).
__device__ __forceinline__ void epi_h16(const GemmParams& p, int b, int row, int col, bool mirror, float f, const float (&v)[32]) {
  if (col >= p.N) return;
  const bool valid = row < p.M;
  __half* dst = p.h_out + b * p.h_batch + (long long)row * p.h_ld + col;
  float w[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) w[j] = f * v[j];
  if (p.aux && valid) {
    const __half* a = p.aux + b * p.h_batch + (long long)row * p.h_ld + col;
#pragma unroll
    for (int pl = 0; pl < 2; ++pl) {
      if (pl && !p.h_plane) break;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint4 q = *reinterpret_cast<const uint4*>(a + pl * p.h_plane + 8 * u);
        const uint32_t x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float lo, hi;
          half2_floats(x[i], lo, hi);
          w[8 * u + 2 * i] = fmaf(p.aux_f, lo, w[8 * u + 2 * i]);
          w[8 * u + 2 * i + 1] = fmaf(p.aux_f, hi, w[8 * u + 2 * i + 1]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (col + j == row) w[j] += p.diag;
  }
  __half hi[32], lo[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) split_half(w[j], hi[j], lo[j]);
#pragma unroll
  for (int pl = 0; pl < 2; ++pl) {
    if (pl && !p.h_plane) break;
    const __half(&h)[32] = pl ? lo : hi;
    if (valid) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        *reinterpret_cast<uint4*>(dst + pl * p.h_plane + 8 * u) =
            make_uint4(pack_half2(h[8 * u], h[8 * u + 1]), pack_half2(h[8 * u + 2], h[8 * u + 3]),
                       pack_half2(h[8 * u + 4], h[8 * u + 5]), pack_half2(h[8 * u + 6], h[8 * u + 7]));
      if (mirror) {   // the lanes hold consecutive rows: 64 bytes of row `col + j` of the mirrored tile
        __half* m = p.h_out + pl * p.h_plane + b * p.h_batch + (long long)col * p.h_ld + row;
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (col + j < p.N) m[(long long)j * p.h_ld] = h[j];
      }
    }
  }
}

// One 32-column group of EPI_OUT: through the warp's scratch, so that a row's 32 values leave in one access whatever the
// row stride of the result (any M, N, alignment of the element type).
__device__ __forceinline__ void epi_out(const GemmParams& p, int b, int row0, int col, float f, const float (&v)[32], float* scratch,
                                        int lane) {
  if (col >= p.N) return;
#pragma unroll
  for (int j = 0; j < 32; ++j) scratch[lane * 33 + j] = f * v[j];
  __syncwarp();
  const int rows = min(32, p.M - row0);
  const bool ok = col + lane < p.N;
  const long long at = (p.use_off ? p.off[b] : b * p.out_batch) + (long long)row0 * p.out_ld + col + lane;
  const long long acc_at = (long long)row0 * p.N + col + lane;
#pragma unroll 8
  for (int r = 0; r < rows; ++r) {
    if (ok) {
      float x = scratch[r * 33 + lane];
      if (p.acc) {
        float* s = p.acc + acc_at + (long long)r * p.N;
        if (!p.acc_first) x += *s;
        if (!p.acc_last) *s = x;
      }
      if (!p.acc || p.acc_last) {
        if (p.out_bf16) {
          bf16* o = (bf16*)p.out + at + (long long)r * p.out_ld;
          if (p.update) x = fmaf(p.step, x, p.keep * __bfloat162float(*o));
          *o = __float2bfloat16_rn(x);
        } else {
          float* o = (float*)p.out + at + (long long)r * p.out_ld;
          if (p.update) x = fmaf(p.step, x, p.keep * *o);
          *o = x;
        }
      }
    }
  }
  __syncwarp();
}

// Logits of a 32-column group: scale, bias, and -inf past the last class.
__device__ __forceinline__ void ce_logits(const GemmParams& p, int col, float f, int lane, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] *= f;
  if (p.bias) {
    float bl = 0.f;
    if (col + lane < p.N) bl = p.bias_bf16 ? __bfloat162float(((const bf16*)p.bias)[col + lane]) : ((const float*)p.bias)[col + lane];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, bl, j);
  }
  if (col + 32 > p.N) {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (col + j >= p.N) v[j] = -INFINITY;
  }
}

constexpr float kLog2e = 1.4426950408889634f;
// Exponentials are kept 2^14 times larger than they are (at most 2^14): fp16 has no 11 bits below 2^-14, and no second part.
constexpr float kCeExpBits = 14.f;

// kPair: tiles of 256 x 256 on CTA pairs, else 128 x 128 on single CTAs.
template <int kEpi, bool kPair, bool kRounds>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_tc_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ GemmParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* scratch_all = reinterpret_cast<float*>(smem + kGemmStages * kGemmStageBytes);
  GemmTail* tail = reinterpret_cast<GemmTail*>(scratch_all + kGemmEpiWarps * kGemmScratchFloats);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kCtas = kPair ? 2 : 1;
  constexpr int kTileM = 128 * kCtas, kTileN = 128 * kCtas;
  constexpr uint32_t kAccCols = kTileN, kTmem = 2 * kAccCols;
  const uint32_t rank = kPair ? cluster_ctarank() : 0;
  const bool leader = rank == 0;
  const int unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kGemmStages; ++s) {
      mbar_init(&tail->full[s], 1);
      mbar_init(&tail->empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&tail->tmem_full[s], 1);
      mbar_init(&tail->tmem_empty[s], kGemmEpiWarps * kCtas);
    }
    tail->abort_flag = 0;
    fence_barrier_init();
    prefetch_tmap(&tmA);
    prefetch_tmap(&tmB);
  }
  if (warp == 2) {
    if constexpr (kPair) {
      tmem2_alloc(&tail->tmem_base, kTmem);
      tmem2_relinquish();
    } else {
      tmem_alloc(&tail->tmem_base, kTmem);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (kPair) cluster_sync_all();   // both CTAs' barriers exist before anything signals them from the other side
  tc_fence_after();
  pdl_wait();
  pdl_launch_dependents();
  const uint32_t tmem_base = tail->tmem_base;
  const int steps = p.kblocks * p.nseg;
  const int round_len = kRounds ? p.round_len : steps;
  bool failed = false;

  if (warp == 0) {
    uint32_t s = 0, ph = 0;
    for (int t = unit; t < p.total_tiles && !failed; t += units) {
      int b, tm, tn;
      gemm_tile(p, t, b, tm, tn);
      const int m0 = tm * kTileM + (int)rank * 128, n0 = tn * kTileN + (int)rank * 128;
      int kb = 0, seg = 0;
      for (int i = 0; i < steps; ++i) {
        if (!mbar_wait_warp(&tail->empty[s], ph ^ 1, abort_flag)) { failed = true; break; }
        if (elect_one()) {
          uint8_t* pa = smem + s * kGemmStageBytes;
          uint8_t* pb = pa + 16384;
          const int az = p.a_z[seg] + b, bz = p.b_z[seg] + b, k0 = kb * 64;
          if constexpr (kPair) {
            const uint32_t fb = mapa_u32(smem_u32(&tail->full[s]), 0);
            if (leader) mbar_expect_tx(&tail->full[s], 2 * kGemmStageBytes);
            if (p.a_mn) {
              tma2_load_3d(pa, &tmA, fb, m0, k0, az);
              tma2_load_3d(pa + 8192, &tmA, fb, m0 + 64, k0, az);
            } else {
              tma2_load_3d(pa, &tmA, fb, k0, m0, az);
            }
            if (p.b_mn) {
              tma2_load_3d(pb, &tmB, fb, n0, k0, bz);
              tma2_load_3d(pb + 8192, &tmB, fb, n0 + 64, k0, bz);
            } else {
              tma2_load_3d(pb, &tmB, fb, k0, n0, bz);
            }
          } else {
            uint64_t* fb = &tail->full[s];
            mbar_expect_tx(fb, kGemmStageBytes);
            if (p.a_mn) {
              tma_load_3d(pa, &tmA, fb, m0, k0, az);
              tma_load_3d(pa + 8192, &tmA, fb, m0 + 64, k0, az);
            } else {
              tma_load_3d(pa, &tmA, fb, k0, m0, az);
            }
            if (p.b_mn) {
              tma_load_3d(pb, &tmB, fb, n0, k0, bz);
              tma_load_3d(pb + 8192, &tmB, fb, n0 + 64, k0, bz);
            } else {
              tma_load_3d(pb, &tmB, fb, k0, n0, bz);
            }
          }
        }
        __syncwarp();
        if (++s == kGemmStages) { s = 0; ph ^= 1; }
        if (++seg == p.nseg) { seg = 0; ++kb; }
      }
    }
  } else if (warp == 1 && leader) {
    // one thread issues (see the MMA issuers of conv_tc_kernel)
    if (elect_one()) {
      // K-major operand: rows of 128 bytes (64 K values), groups of 8 rows 1024 bytes apart, 16 K values further = 32 bytes.
      // Row-contiguous operand: two boxes of 64 rows, K down the box: 16 K values further = 16 lines of 128 bytes.
      const uint64_t da = p.a_mn ? smem_desc_hi(8192, 1024, 2) : smem_desc_hi(16, 1024, 2);
      const uint64_t db = p.b_mn ? smem_desc_hi(8192, 1024, 2) : smem_desc_hi(16, 1024, 2);
      const uint32_t ka = p.a_mn ? 128 : 2, kb16 = p.b_mn ? 128 : 2;
      const uint32_t base = smem_u32(smem);
      uint32_t s = 0, ph = 0, buf = 0, bph = 0;
      for (int t = unit; t < p.total_tiles && !failed; t += units) {
        for (int i0 = 0; i0 < steps && !failed; i0 += round_len) {
          if (!mbar_wait_hot(&tail->tmem_empty[buf], bph ^ 1, abort_flag)) { failed = true; break; }
          tc_fence_after();
          const uint32_t d = tmem_base + buf * kAccCols;
          const int i1 = min(steps, i0 + round_len);
#pragma unroll 1
          for (int i = i0; i < i1; ++i) {
            if (!mbar_wait_hot(&tail->full[s], ph, abort_flag)) { failed = true; break; }
            tc_fence_after();
            const uint64_t ad = smem_desc(da, base + s * kGemmStageBytes), bd = smem_desc(db, base + s * kGemmStageBytes + 16384);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (kPair) mma2_bf16(d, ad + (uint64_t)(j * ka), bd + (uint64_t)(j * kb16), p.idesc, (i > i0 || j) ? 1u : 0u);
              else mma_bf16(d, ad + (uint64_t)(j * ka), bd + (uint64_t)(j * kb16), p.idesc, (i > i0 || j) ? 1u : 0u);
            }
            if constexpr (kPair) mma2_commit_both(&tail->empty[s]);
            else mma_commit(&tail->empty[s]);
            if (++s == kGemmStages) { s = 0; ph ^= 1; }
          }
          if (failed) break;
          if constexpr (kPair) mma2_commit_both(&tail->tmem_full[buf]);
          else mma_commit(&tail->tmem_full[buf]);
          buf ^= 1;
          if (!buf) bph ^= 1;
        }
      }
    }
    __syncwarp();
    failed = __any_sync(0xffffffffu, failed);
  } else if (warp >= 2) {
    const int q = warp & 3, half = (warp - 2) >> 2;
    constexpr int kGroups = kTileN / 64;       // 32-column groups of this warp's half
    float* scratch = scratch_all + (warp - 2) * kGemmScratchFloats;
    uint32_t buf = 0, bph = 0;
    for (int t = unit; t < p.total_tiles && !failed; t += units) {
      int b, tm, tn;
      gemm_tile(p, t, b, tm, tn);
      const int row0 = tm * kTileM + (int)rank * 128 + q * 32, row = row0 + lane;
      const int col0 = tn * kTileN + half * (kTileN / 2);
      const float f = gemm_scale(p, b);
      float acc[kRounds ? kGroups : 1][32];
      if constexpr (kRounds) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int j = 0; j < 32; ++j) acc[g][j] = 0.f;
      }
      for (int i0 = 0; i0 < steps; i0 += round_len) {
        if (!mbar_wait_warp(&tail->tmem_full[buf], bph, abort_flag)) { failed = true; break; }
        tc_fence_after();
        const uint32_t taddr = tmem_base + buf * kAccCols + half * (kTileN / 2) + ((uint32_t)(q * 32) << 16);
        auto release = [&] {   // everything of this accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (kPair) mbar_arrive_cluster(mapa_u32(smem_u32(&tail->tmem_empty[buf]), 0));
            else mbar_arrive(&tail->tmem_empty[buf]);
          }
        };
        if constexpr (kRounds) {
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            float v[32];
            tmem_ld32(taddr + g * 32, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[g][j] += v[j];
          }
          release();
        }
        if (!kRounds || i0 + round_len >= steps) {
          if constexpr (kEpi == EPI_CE) {
            float top = -INFINITY;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              float v[32];
              if constexpr (!kRounds) tmem_ld32(taddr + g * 32, v);
              else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = acc[g][j];
              }
              ce_logits(p, col0 + g * 32, f, lane, v);
#pragma unroll
              for (int j = 0; j < 32; ++j) top = fmaxf(top, v[j]);
            }
            const float ref = top == -INFINITY ? 0.f : top;   // a half without any class counts nothing
            const int label = row < p.M ? p.labels[row] : -1;
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              const int col = col0 + g * 32;
              float v[32];
              if constexpr (!kRounds) tmem_ld32(taddr + g * 32, v);
              else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = acc[g][j];
              }
              if constexpr (!kRounds) {
                if (g + 1 == kGroups) release();
              }
              ce_logits(p, col, f, lane, v);
              if (label >= col && label < col + 32) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (col + j == label) p.target[row] = v[j];
              }
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                v[j] = exp2f(fmaf(v[j] - ref, kLog2e, kCeExpBits));
                sum += v[j];
              }
              if (p.h_out && row < p.M && col < p.N) {
                __half* dst = p.h_out + (long long)row * p.h_ld + col;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  __half hi[8], lo[8];
#pragma unroll
                  for (int j = 0; j < 8; ++j) split_half(v[8 * u + j], hi[j], lo[j]);
                  *reinterpret_cast<uint4*>(dst + 8 * u) = make_uint4(pack_half2(hi[0], hi[1]), pack_half2(hi[2], hi[3]),
                                                                      pack_half2(hi[4], hi[5]), pack_half2(hi[6], hi[7]));
                  if (kRounds)
                    *reinterpret_cast<uint4*>(dst + p.h_plane + 8 * u) = make_uint4(pack_half2(lo[0], lo[1]), pack_half2(lo[2], lo[3]),
                                                                                    pack_half2(lo[4], lo[5]), pack_half2(lo[6], lo[7]));
                }
              }
            }
            if (row < p.M) p.stats[(long long)(tn * 2 + half) * p.stats_ld + row] = make_float2(ref, sum * 6.103515625e-5f);
          } else {
            const bool mirror = p.sym && tm != tn;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              float v[32];
              if constexpr (!kRounds) {
                tmem_ld32(taddr + g * 32, v);
                if (g + 1 == kGroups) release();
              } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = acc[g][j];
              }
              if constexpr (kEpi == EPI_H16) epi_h16(p, b, row, col0 + g * 32, mirror, f, v);
              else epi_out(p, b, row0, col0 + g * 32, f, v, scratch, lane);
            }
          }
        }
        buf ^= 1;
        if (!buf) bph ^= 1;
      }
    }
  }

  if (failed) {
    *abort_flag = 1;
    atomicExch(p.err, 1);
    // let copies and MMAs already in flight land before shared / tensor memory is released
#pragma unroll 1
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag && !failed) {
#pragma unroll 1
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  if constexpr (kPair) cluster_sync_all();   // neither CTA leaves while the other may still signal it
  if (warp == 2) {
    tc_fence_after();
    if constexpr (kPair) tmem2_dealloc(tmem_base, kTmem);
    else tmem_dealloc(tmem_base, kTmem);
  }
}

}  // namespace tc
}  // namespace lp
