// Dense batched matrix products on the tensor cores for the operators at the end of a training step (linear_ce.cuh,
// ortho.cuh): D[b] = A[b] B[b]^T with 16-bit operands and fp32 accumulation, each operand stored with either dimension
// contiguous, and the operator's own arithmetic in the epilogue.
//
// Tiles.  A CTA pair (cta_group::2) computes 256 x 256: each CTA holds 128 rows of A and 128 of B's 256 rows, and every
// tcgen05.mma reads both halves, so a 64-wide K block costs an SM 32 KB of loads for 128 x 256 x 64 products -- 64 bytes a
// cycle, what an SM draws from L2.  Products with too few such tiles to fill the SMs take 128 x 128 tiles on single CTAs, and
// products in two parts where it leaves fewer SMs idle 256 x 128 tiles on pairs.
// The grid is persistent: a CTA (pair) walks the tiles, six stages of operands in flight, two accumulators in tensor
// memory, so that a tile's epilogue runs under the next tile's products.
//
// Precision.  Operands may be kept as a 16-bit high and a low part (planes of the same tensor): a stage holds all planes of
// its K block, and hi*hi + hi*lo + lo*hi go into one accumulation (four tiles fetched for three products; lo*lo is below what
// the parts keep).  Where fp32 results are wanted (kRounds), the tensor core's accumulator is emptied every `round_len` K
// blocks into registers and added up there: the accumulation inside the tensor core does not round to nearest, and its error
// grows with the number of K steps.
//
// Roles (320 threads): warp 0 TMA producer, warp 1 MMA issuer (of the pair's leader), warps 2..9 epilogue: two warps per
// quarter of the accumulator's rows, each taking one half of its columns; a thread has one row.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace lp {
namespace tc {

constexpr int kGemmStages = 6;                 // at most: 6 of one plane of each operand, 4 of three planes, 3 of four
constexpr int kGemmThreads = 320;
constexpr int kGemmEpiWarps = 8;
constexpr uint32_t kGemmTileBytes = 16384;    // 128 rows x 64 columns of a plane, 16 bits each
constexpr uint32_t kGemmRingBytes = 12 * kGemmTileBytes;
constexpr int kGemmScratchFloats = 32 * 33;   // per epilogue warp: a 32 x 32 block, written row by row where rows are not aligned
constexpr int kGemmMaxOffsets = 64;

struct GemmTail {
  uint64_t full[kGemmStages], empty[kGemmStages];
  uint64_t tmem_full[2], tmem_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};
constexpr size_t kGemmSmem = 1024 + (size_t)kGemmRingBytes + (size_t)kGemmEpiWarps * kGemmScratchFloats * 4 + sizeof(GemmTail);
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
  int kblocks;
  int a_planes, b_planes;         // parts of each operand (1 or 2), `batch` matrices apart
  int round_len;                  // kRounds: K blocks per accumulation (0: see launch_gemm)
  int a_mn, b_mn;                 // 1: the operand's row index is the contiguous one
  uint32_t idesc;
  // Two products side by side that read the same operands and write different results: the first (`publish` given) stores `turn`
  // there once it has waited for the kernels before it, and before it lets the second start; the second (`wait_late`) acquires that
  // word, by which it sees all that the first saw, and waits for the first one's end before its own.  (A grid's own wait is all
  // that orders it behind the grids before, so starting without one needs the word; if it is not there yet, it waits after all.
  // A call clears the word in a kernel that both follow.)
  int* publish;
  const int* wait_late;
  int turn;
  int* err;
  int* clear;                     // two words (the error word is the first) to clear, or null
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
  int out_bf16, out_vec;          // out_vec: every row of out (and acc) starts on 32 bytes and N is a multiple of 32 bytes
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
  const int32_t* labels;          // [M]; EPI_OUT: rows whose label is none of `classes` are written as zeros (or null)
  int classes;
  float2* stats;                  // [part of the columns][M]: maximum, sum of exponentials
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
__device__ __forceinline__ void half2_floats(uint32_t u, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
  a = f.x;
  b = f.y;
}
// Two at once (one instruction; converting one value at a time runs at an eighth of the rate).
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Both parts of two values.
__device__ __forceinline__ void split_f16x2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_f16x2(a, b);
  float ha, hb;
  half2_floats(hi, ha, hb);
  lo = pack_f16x2(a - ha, b - hb);
}

// 32-byte global accesses (addresses are 32-byte aligned): a thread has a row of the accumulator, and what it reads or writes of
// 32 columns there goes by whole sectors.  Not through shared memory: at 64 bytes a cycle written by the loads and 64 read by
// the products, the rings leave none of its bandwidth (a pass through scratch cost the mainloop 10 % at K = 2048).
__device__ __forceinline__ void st_v8(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void st_v8f(float* p, const float* v) {
  const uint32_t u[8] = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]),
                         __float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
  st_v8(p, u);
}
__device__ __forceinline__ void ld_v8(const void* p, uint32_t* v) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "l"(p)
               : "memory");
}

// One 32-column group of an intermediate, as fp16 planes, by a whole warp; `row` is the lane's, row0 < M the warp's first.  Columns
// past N are written as far as the buffer's rows are padded (whole groups of 32); what lies there is never read.  `mirror`: the
// block above the diagonal of a symmetric result goes below it, too, turned over in the warp's scratch: the lanes then hold rows of
// the mirrored block (stored by twos from where they are, 32 accesses of 64 bytes a group made the tile's end 2 us later).
__device__ __forceinline__ void epi_h16(const GemmParams& p, int b, int row0, int lane, int col, bool mirror, float (&v)[32], float* scratch) {
  const int row = row0 + lane;
  const bool valid = row < p.M;
  const long long at = b * p.h_batch + (long long)row * p.h_ld + col;
  if (p.aux && valid) {
#pragma unroll
    for (int pl = 0; pl < 2; ++pl) {
      if (pl && !p.h_plane) break;
      uint32_t x[16];
      ld_v8(p.aux + pl * p.h_plane + at, x);
      ld_v8(p.aux + pl * p.h_plane + at + 16, x + 8);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float lo, hi;
        half2_floats(x[i], lo, hi);
        v[2 * i] = fmaf(p.aux_f, lo, v[2 * i]);
        v[2 * i + 1] = fmaf(p.aux_f, hi, v[2 * i + 1]);
      }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (col + j == row) v[j] += p.diag;
  }
#pragma unroll
  for (int pl = 0; pl < 2; ++pl) {
    if (pl && !p.h_plane) break;
    __half* out = p.h_out + pl * p.h_plane;
    uint32_t h[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      h[i] = pack_f16x2(v[2 * i], v[2 * i + 1]);
      if (p.h_plane) {       // what is left for the low part
        float x, y;
        half2_floats(h[i], x, y);
        v[2 * i] -= x;
        v[2 * i + 1] -= y;
      }
    }
    if (valid) {
      st_v8(out + at, h);
      st_v8(out + at + 16, h + 8);
    }
    if (mirror) {
      uint32_t* t = reinterpret_cast<uint32_t*>(scratch);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 16; ++i) t[lane * 17 + i] = h[i];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 16; ++i)   // column `lane` of rows 2 i and 2 i + 1
        h[i] = __byte_perm(t[2 * i * 17 + (lane >> 1)], t[(2 * i + 1) * 17 + (lane >> 1)], lane & 1 ? 0x7632 : 0x5410);
      if (col + lane < p.N) {
        __half* m = out + b * p.h_batch + (long long)(col + lane) * p.h_ld + row0;
        st_v8(m, h);
        st_v8(m + 16, h + 8);
      }
    }
  }
}

// One 32-column group of a result in the caller's type whose rows are 32-byte aligned (and N a multiple of 32 bytes of it).
// What is added to, or updated, is read before anything is written: its reads are in flight together.
__device__ __forceinline__ void epi_out_vec(const GemmParams& p, int b, int row, int col, float (&v)[32]) {
  if (row >= p.M) return;
  const int n = min(32, p.N - col);
  if (p.acc) {
    float* acc = p.acc + (long long)row * p.N + col;
    if (!p.acc_first) {
      uint32_t x[32];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (8 * u < n) ld_v8(acc + 8 * u, x + 8 * u);
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < n) v[j] += __uint_as_float(x[j]);
    }
    if (!p.acc_last) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (8 * u < n) st_v8f(acc + 8 * u, v + 8 * u);
      return;
    }
  }
  const long long at = (p.use_off ? p.off[b] : b * p.out_batch) + (long long)row * p.out_ld + col;
  if (p.out_bf16) {
    bf16* o = (bf16*)p.out + at;
    uint32_t x[16];
    if (p.update) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (16 * u < n) ld_v8(o + 16 * u, x + 8 * u);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[2 * i] = fmaf(p.step, v[2 * i], p.keep * __uint_as_float(x[i] << 16));
        v[2 * i + 1] = fmaf(p.step, v[2 * i + 1], p.keep * __uint_as_float(x[i] & 0xFFFF0000u));
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (16 * u < n) st_v8(o + 16 * u, x + 8 * u);
  } else {
    float* o = (float*)p.out + at;
    if (p.update) {
      uint32_t x[32];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (8 * u < n) ld_v8(o + 8 * u, x + 8 * u);
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = fmaf(p.step, v[j], p.keep * __uint_as_float(x[j]));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (8 * u < n) st_v8f(o + 8 * u, v + 8 * u);
  }
}

// The same for any row stride: through the warp's scratch, so that a row's 32 values leave in one access.  Eight rows at a
// time: their reads are in flight together.
template <typename T>
__device__ __forceinline__ void rows_to(T* out, long long ld, int rows, float* scratch, bool add, float keep, float step) {
#pragma unroll 1
  for (int r = 0; r < rows; r += 8) {
    if (add) {
      T old[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + i < rows) old[i] = out[(r + i) * ld];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + i < rows) from_f(out[(r + i) * ld], fmaf(step, scratch[(r + i) * 33], keep * to_f(old[i])));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + i < rows) from_f(out[(r + i) * ld], scratch[(r + i) * 33]);
    }
  }
}
__device__ __forceinline__ void epi_out_any(const GemmParams& p, int b, int row0, int col, const float (&v)[32], float* scratch, int lane) {
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 32; ++j) scratch[lane * 33 + j] = v[j];
  __syncwarp();
  if (col + lane >= p.N) return;
  const int rows = min(32, p.M - row0);
  scratch += lane;
  if (p.acc) {
    float* acc = p.acc + (long long)row0 * p.N + col + lane;
    rows_to(acc, p.N, rows, scratch, !p.acc_first, 1.f, 1.f);
    if (!p.acc_last) return;
    for (int r = 0; r < rows; ++r) scratch[r * 33] = acc[(long long)r * p.N];   // (this lane's own sums)
  }
  const long long at = (p.use_off ? p.off[b] : b * p.out_batch) + (long long)row0 * p.out_ld + col + lane;
  if (p.out_bf16) rows_to((bf16*)p.out + at, p.out_ld, rows, scratch, p.update, p.keep, p.step);
  else rows_to((float*)p.out + at, p.out_ld, rows, scratch, p.update, p.keep, p.step);
}

// Logits of a 32-column group: scale, bias (lane j's `bias` is of column `col` + j), and -inf past the last class.
__device__ __forceinline__ void ce_logits(const GemmParams& p, int col, float f, float bias, float (&v)[32]) {
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = fmaf(f, v[j], __shfl_sync(0xffffffffu, bias, j));
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] *= f;
  }
  if (col + 32 > p.N) {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (col + j >= p.N) v[j] = -INFINITY;
  }
}
__device__ __forceinline__ float ce_bias(const GemmParams& p, int col) {
  if (!p.bias || col >= p.N) return 0.f;
  return p.bias_bf16 ? __bfloat162float(((const bf16*)p.bias)[col]) : ((const float*)p.bias)[col];
}

// bias[g], in registers
template <int N>
__device__ __forceinline__ float ce_pick(const float (&bias)[N], int g) {
  float v = bias[0];
#pragma unroll
  for (int i = 1; i < N; ++i) v = g == i ? bias[i] : v;
  return v;
}

constexpr float kLog2e = 1.4426950408889634f;
// Exponentials are kept 2^14 times larger than they are (at most 2^14): fp16 has no 11 bits below 2^-14, and no second part.
constexpr float kCeExpBits = 14.f;

// What a K block's stage holds, and whether the accumulator is emptied in rounds.
enum GemmMode {
  GEMM_ONE = 0,      // one plane of each operand
  GEMM_LOW = 1,      // a low part of one operand, too
  GEMM_SPLIT = 2,    // both parts of both, in rounds
  GEMM_LONG = 3,     // one plane of each, in rounds (a long K whose sum is wanted in fp32)
};

// How a tile is computed.
enum GemmKind {
  GEMM_SINGLE = 0,   // 128 x 128 by one CTA
  GEMM_PAIR = 1,     // 256 x 256 by a CTA pair
  GEMM_KSPLIT = 2,   // 128 x 128 by a cluster of 2, 3, 4 or 8 CTAs, a share of K each; one tile a cluster
  GEMM_HALF = 3,     // 256 x 128 by a CTA pair (GEMM_SPLIT: with three products a K block its loads keep up)
};

template <int kEpi, int kKind, int kMode>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_tc_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ GemmParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* scratch_all = reinterpret_cast<float*>(smem + kGemmRingBytes);
  GemmTail* tail = reinterpret_cast<GemmTail*>(scratch_all + kGemmEpiWarps * kGemmScratchFloats);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr bool kHalf = kKind == GEMM_HALF, kPair = kKind == GEMM_PAIR || kHalf, kKSplit = kKind == GEMM_KSPLIT;
  static_assert(!kHalf || kMode == GEMM_SPLIT, "stages below");
  constexpr int kCtas = kPair ? 2 : 1;
  constexpr bool kCluster = kPair || kKSplit;
  constexpr int kTileM = 128 * kCtas, kTileN = kHalf ? 128 : 128 * kCtas;
  constexpr uint32_t kRowsB = kTileN / kCtas, kTileBytesB = kRowsB * 128;   // of B, of a plane in a stage
  constexpr uint32_t kAccCols = kTileN, kTmem = 2 * kAccCols;
  const uint32_t crank = kCluster ? cluster_ctarank() : 0;
  const uint32_t rank = kPair ? crank : 0;      // of the CTAs that share a tile's rows
  const bool leader = rank == 0;
  const int ctas = kKSplit ? (int)cluster_nctas() : kCtas;
  const int unit = blockIdx.x / ctas, units = gridDim.x / ctas;

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
  if constexpr (kCluster) cluster_sync_all();   // both CTAs' barriers exist before anything signals them from the other side
  tc_fence_after();
  if (!p.wait_late || ld_acquire(p.wait_late) != p.turn) pdl_wait();
  if (p.wait_late) fence_async_global();   // (what was written before is read through TMA)
  if (p.publish && blockIdx.x == 0 && threadIdx.x == 0) st_release(p.publish, p.turn);
  if (p.clear && blockIdx.x == 0 && threadIdx.x == 0) p.clear[0] = p.clear[1] = 0;   // (a wait gives up after 0.3 s at the earliest)
  pdl_launch_dependents();
  const uint32_t tmem_base = tail->tmem_base;
  // (its share of K: at least one K block, see gemm_cut)
  const int k_first = kKSplit ? p.kblocks * (int)crank / ctas : 0;
  const int steps = kKSplit ? p.kblocks * (int)(crank + 1) / ctas - k_first : p.kblocks;
  constexpr bool kRounds = kMode == GEMM_SPLIT || kMode == GEMM_LONG;
  const int round_len = kRounds ? p.round_len : steps;
  constexpr uint32_t kTiles = kMode == GEMM_SPLIT ? 4 : kMode == GEMM_LOW ? 3 : 2;
  constexpr uint32_t kStages = kHalf ? 4 : 12 / kTiles;
  constexpr uint32_t kStageBytes = kHalf ? 2 * (kGemmTileBytes + kTileBytesB) : kTiles * kGemmTileBytes;
  static_assert(kStages <= kGemmStages && kStages * kStageBytes <= kGemmRingBytes, "the ring");
  // (GEMM_LOW: which operand has two parts is known at run time)
  const int a_planes = kMode == GEMM_SPLIT ? 2 : (kMode == GEMM_LOW ? p.a_planes : 1);
  bool failed = false;

  if (warp == 0) {
    uint32_t s = 0, ph = 0;
    for (int t = unit; t < p.total_tiles && !failed; t += units) {
      int b, tm, tn;
      gemm_tile(p, t, b, tm, tn);
      const int m0 = tm * kTileM + (int)rank * 128, n0 = tn * kTileN + (int)(rank * kRowsB);
      for (int i = 0; i < steps; ++i) {
        if (!mbar_wait_warp(&tail->empty[s], ph ^ 1, abort_flag)) { failed = true; break; }
        if (elect_one()) {
          uint8_t* dst = smem + s * kStageBytes;
          const int k0 = (k_first + i) * 64;
          uint64_t* full = &tail->full[s];
          const uint32_t fb = kPair ? mapa_u32(smem_u32(full), 0) : 0;
          if (leader) mbar_expect_tx(full, kCtas * kStageBytes);
#pragma unroll
          for (int x = 0; x < (int)kTiles; ++x) {
            const bool is_a = x < a_planes;
            const CUtensorMap* map = is_a ? &tmA : &tmB;
            const int r0 = is_a ? m0 : n0, z = (is_a ? x : x - a_planes) * p.batch + b;
            // rows contiguous: boxes of 64 rows by 64 K; K contiguous: one of all rows
            if (is_a ? p.a_mn : p.b_mn) {
              if constexpr (kPair) {
                tma2_load_3d(dst, map, fb, r0, k0, z);
                if (is_a || !kHalf) tma2_load_3d(dst + 8192, map, fb, r0 + 64, k0, z);
              } else {
                tma_load_3d(dst, map, full, r0, k0, z);
                tma_load_3d(dst + 8192, map, full, r0 + 64, k0, z);
              }
            } else {
              if constexpr (kPair) tma2_load_3d(dst, map, fb, k0, r0, z);
              else tma_load_3d(dst, map, full, k0, r0, z);
            }
            dst += is_a ? kGemmTileBytes : kTileBytesB;
          }
        }
        __syncwarp();
        if (++s == kStages) { s = 0; ph ^= 1; }
      }
    }
    if constexpr (kPair) {   // what the leader's products signal has arrived before this CTA leaves (the last barrier orders nothing)
      for (uint32_t i = 0; i < kStages && !failed; ++i) {
        failed = !mbar_wait_warp(&tail->empty[s], ph ^ 1, abort_flag);
        if (++s == kStages) { s = 0; ph ^= 1; }
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
            const uint32_t at = base + s * kStageBytes;
            auto product = [&](int x, int y, uint32_t more) {   // tiles x (of A) and y (of B) of the stage
              const uint32_t of_b = kHalf ? 2 * kGemmTileBytes + (y - 2) * kTileBytesB : y * kGemmTileBytes;
              const uint64_t ad = smem_desc(da, at + x * kGemmTileBytes), bd = smem_desc(db, at + of_b);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if constexpr (kPair) mma2_bf16(d, ad + (uint64_t)(j * ka), bd + (uint64_t)(j * kb16), p.idesc, j ? 1u : more);
                else mma_bf16(d, ad + (uint64_t)(j * ka), bd + (uint64_t)(j * kb16), p.idesc, j ? 1u : more);
              }
            };
            // low parts first: the accumulator is cut off at each step, by less while it is small
            const uint32_t more = i > i0 ? 1u : 0u;
            if constexpr (kMode == GEMM_SPLIT) {
              product(0, 3, more);
              product(1, 2, 1u);
              product(0, 2, 1u);
            } else if constexpr (kMode == GEMM_LOW) {
              product(a_planes - 1, 2, more);
              product(0, a_planes == 2 ? 2 : 1, 1u);
            } else {
              product(0, 1, more);
            }
            if constexpr (kPair) mma2_commit_both(&tail->empty[s]);
            else mma_commit(&tail->empty[s]);
            if (++s == kStages) { s = 0; ph ^= 1; }
          }
          if (failed) break;
          if constexpr (kPair) mma2_commit_both(&tail->tmem_full[buf]);
          else mma_commit(&tail->tmem_full[buf]);
          buf ^= 1;
          if (!buf) bph ^= 1;
        }
      }
      if constexpr (kPair) {   // and what the other CTA's epilogue signals has arrived here
        for (int i = 0; i < 2 && !failed; ++i) {
          failed = !mbar_wait_hot(&tail->tmem_empty[buf], bph ^ 1, abort_flag);
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
      int col0 = tn * kTileN + half * (kTileN / 2);
      const float f = gemm_scale(p, b);
      // (read while the products are under way)
      float bias[kGroups] = {};
      int label = -1;
      // (a select, not a product: what stands there may be no number)
      bool zero_row = false;
      if constexpr (kEpi == EPI_OUT) {
        if (p.labels && row < p.M) {
          label = p.labels[row];
          zero_row = label < 0 || label >= p.classes;
        }
      }
      if constexpr (kEpi == EPI_CE) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) bias[g] = ce_bias(p, col0 + g * 32 + lane);
        if (row < p.M) label = p.labels[row];
      }
      float acc[kRounds ? kGroups : 1][32];
      if constexpr (kRounds) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int j = 0; j < 32; ++j) acc[g][j] = 0.f;
      }
      uint32_t taddr;
      auto release = [&] {   // everything of this accumulator has been read
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair) mbar_arrive_cluster_relaxed(mapa_u32(smem_u32(&tail->tmem_empty[buf]), 0));
          else mbar_arrive(&tail->tmem_empty[buf]);
        }
      };
      for (int i0 = 0;; i0 += round_len) {
        if (!mbar_wait_warp(&tail->tmem_full[buf], bph, abort_flag)) { failed = true; break; }
        tc_fence_after();
        taddr = tmem_base + buf * kAccCols + half * (kTileN / 2) + ((uint32_t)(q * 32) << 16);
        if constexpr (kRounds) {
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            float v[32];
            tmem_ld32(taddr + g * 32, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[g][j] += v[j];
          }
        }
        if (i0 + round_len >= steps) break;
        release();
        buf ^= 1;
        if (!buf) bph ^= 1;
      }
      if (failed && !kKSplit) break;
      int groups = kGroups;
      if constexpr (kRounds) {   // the sum goes back to where the accumulator was: what follows reads it group by group
        if (!failed) {
#pragma unroll
          for (int g = 0; g < kGroups; ++g) tmem_st32(taddr + g * 32, acc[g]);
        }
      }
      if constexpr (kKSplit) {
        // Group g of 32 columns is finished by CTA g % c.  Every CTA leaves the groups of the others in its own shared memory (over
        // the ring: all its products have read it), four columns of 128 rows together; after the barrier the warps that have the
        // CTA's group fetch it from each of the others, 512 bytes in a row an access (16 bytes at a time from rows apart took
        // twice as long as anything else here), and add up, in the CTAs' order.
        float4* ring = reinterpret_cast<float4*>(smem);
        const int c = (int)cluster_nctas();
        int mine = -1;
#pragma unroll 1
        for (int g = 0; g < kGroups; ++g) {
          const int grp = half * kGroups + g;
          if (grp % c == (int)crank) {
            mine = g;
          } else if (!failed) {
            float v[32];
            tmem_ld32(taddr + g * 32, v);
            float4* to = ring + grp * 8 * 128 + q * 32 + lane;
#pragma unroll
            for (int j = 0; j < 8; ++j) to[j * 128] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          }
        }
        __syncwarp();
        cluster_sync_all();
        if (failed || mine < 0) break;
        taddr += mine * 32;
        const uint32_t from = smem_u32(ring + (half * kGroups + mine) * 8 * 128 + q * 32 + lane);
        col0 += mine * 32;
        if (mine) bias[0] = bias[kGroups - 1];
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = 0.f;
#pragma unroll 1
        for (int r = 0; r < c; ++r) {
          float x[32];
          if (r == (int)crank) {
            tmem_ld32(taddr, x);
          } else {
            const uint32_t at = mapa_u32(from, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float4 f = ld_cluster_f32x4(at + j * 2048);
              x[4 * j] = f.x; x[4 * j + 1] = f.y; x[4 * j + 2] = f.z; x[4 * j + 3] = f.w;
            }
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += x[j];
        }
        tmem_st32(taddr, v);
        groups = 1;
      }
      if constexpr (kEpi == EPI_CE) {
        float top = -INFINITY;
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
          float v[32];
          tmem_ld32(taddr + g * 32, v);
          ce_logits(p, col0 + g * 32, f, ce_pick(bias, g), v);
#pragma unroll
          for (int j = 0; j < 32; ++j) top = fmaxf(top, v[j]);
        }
        // (a half without any class: its exponentials are 0, and `stats` says -inf, so that what they are multiplied by later is
        // 0, too, however low the row's lse is)
        const float ref = top == -INFINITY ? 0.f : top;
        float sums[4] = {0.f, 0.f, 0.f, 0.f};   // (a fourth of the roundings of one chain, next to the largest term, 1)
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
          const int col = col0 + g * 32;
          float v[32];
          tmem_ld32(taddr + g * 32, v);
          if (g + 1 == groups) release();
          ce_logits(p, col, f, ce_pick(bias, g), v);
          if (label >= col && label < col + 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (col + j == label) p.target[row] = v[j];
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            v[j] = exp2f(fmaf(v[j] - ref, kLog2e, kCeExpBits));
            sums[j & 3] += v[j];
          }
          if (p.h_out && col < p.N && row0 < p.M) epi_h16(p, 0, row0, lane, col, false, v, scratch);
        }
        const float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        if (row < p.M) p.stats[(long long)(col0 / (kKSplit ? 32 : kTileN / 2)) * p.stats_ld + row] = make_float2(top, sum * 6.103515625e-5f);
      } else {
        const bool mirror = p.sym && tm != tn;
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
          const int col = col0 + g * 32;
          float v[32];
          tmem_ld32(taddr + g * 32, v);
          if (g + 1 == groups) release();
          if (col >= p.N || row0 >= p.M) continue;
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = zero_row ? 0.f : v[j] * f;
          if constexpr (kEpi == EPI_H16) epi_h16(p, b, row0, lane, col, mirror, v, scratch);
          else if (p.out_vec) epi_out_vec(p, b, row, col, v);
          else epi_out_any(p, b, row0, col, v, scratch, lane);
        }
      }
      buf ^= 1;
      if (!buf) bph ^= 1;
    }
  }

  if constexpr (kKSplit) {
    if (warp < 2) {   // the barrier of the exchange is for every thread
      __syncwarp();
      cluster_sync_all();
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
  if (p.wait_late) pdl_wait();
  if constexpr (kCluster) cluster_sync_relaxed();   // no CTA leaves while another may still signal it or read its ring
  if (warp == 2) {
    tc_fence_after();
    if constexpr (kPair) tmem2_dealloc(tmem_base, kTmem);
    else tmem_dealloc(tmem_base, kTmem);
  }
}

}  // namespace tc
}  // namespace lp
