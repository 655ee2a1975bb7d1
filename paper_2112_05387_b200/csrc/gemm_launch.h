// Host side of gemm_tc.cuh: operand descriptions, tile choice, launch.
#pragma once
#include <string.h>

#include <algorithm>

#include "device.h"
#include "gemm_tc.cuh"

namespace lp {

// A 16-bit operand: `planes` x `batch` matrices (batch innermost) of `outer` rows of `inner` contiguous elements, rows `ld`
// elements apart (a multiple of 8, the base 16-byte aligned), matrices `stride` elements apart.
struct GemmOperand {
  const void* p;
  long long inner, outer, ld, stride;
  int count;   // planes * batch
  bool bf16;
};

// `mn`: the operand's row index is the contiguous one (boxes of 64 rows x 64 K), else K is (`rows` x 64 K: 128, or what
// rows_b says for the second operand).
static int encode_gemm_map(CUtensorMap* m, const GemmOperand& o, bool mn, unsigned rows = 128) {
  cuuint64_t dims[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)o.count};
  cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.stride * 2};
  cuuint32_t box[3] = {64, mn ? 64u : rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  CUresult r = cur_dev().encode(m, o.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                            const_cast<void*>(o.p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? LP_OK : LP_ERR_CUDA;
}

template <int kEpi, int kMode>
static int gemm_set_attributes() {
  using namespace tc;
  LP_CUDA_OK(cudaFuncSetAttribute(gemm_tc_kernel<kEpi, GEMM_SINGLE, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGemmSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(gemm_tc_kernel<kEpi, GEMM_PAIR, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGemmSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(gemm_tc_kernel<kEpi, GEMM_KSPLIT, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGemmSmem));
  if constexpr (kMode == GEMM_SPLIT)
    LP_CUDA_OK(cudaFuncSetAttribute(gemm_tc_kernel<kEpi, GEMM_HALF, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGemmSmem));
  return LP_OK;
}
// Clusters of `ctas` CTAs of a kernel that the device holds at once (0: none, or it cannot say).
template <typename... KArgs>
static int max_clusters(int ctas, void (*kernel)(KArgs...), int threads, size_t smem, int sms) {
  cudaLaunchConfig_t q = {};
  q.gridDim = dim3(ctas * sms);
  q.blockDim = dim3(threads);
  q.dynamicSmemBytes = smem;
  cudaLaunchAttribute qa[1];
  qa[0].id = cudaLaunchAttributeClusterDimension;
  qa[0].val.clusterDim.x = ctas; qa[0].val.clusterDim.y = 1; qa[0].val.clusterDim.z = 1;
  q.attrs = qa;
  q.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &q) != cudaSuccess) { cudaGetLastError(); n = 0; }
  return n;
}
// Sizes of the clusters that share K.
static const int kKShares[] = {2, 3, 4, 8};
// Kernel attributes, and how many CTA pairs the device holds at once (the grid is persistent: never more than that).
static int gemm_init_dev() {
  int rc = init_cur_dev();
  if (rc != LP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_devices_mutex);
  Device& D = cur_dev();
  if (D.gemm_attr) return LP_OK;
  using namespace tc;
  if ((rc = gemm_set_attributes<EPI_H16, GEMM_ONE>()) != LP_OK || (rc = gemm_set_attributes<EPI_H16, GEMM_LOW>()) != LP_OK ||
      (rc = gemm_set_attributes<EPI_H16, GEMM_SPLIT>()) != LP_OK || (rc = gemm_set_attributes<EPI_OUT, GEMM_ONE>()) != LP_OK ||
      (rc = gemm_set_attributes<EPI_OUT, GEMM_LOW>()) != LP_OK || (rc = gemm_set_attributes<EPI_OUT, GEMM_SPLIT>()) != LP_OK ||
      (rc = gemm_set_attributes<EPI_CE, GEMM_ONE>()) != LP_OK || (rc = gemm_set_attributes<EPI_CE, GEMM_SPLIT>()) != LP_OK ||
      (rc = gemm_set_attributes<EPI_CE, GEMM_LONG>()) != LP_OK || (rc = gemm_set_attributes<EPI_H16, GEMM_LONG>()) != LP_OK ||
      (rc = gemm_set_attributes<EPI_OUT, GEMM_LONG>()) != LP_OK)
    return rc;
  D.gemm_pairs = max_clusters(2, gemm_tc_kernel<EPI_OUT, GEMM_PAIR, GEMM_ONE>, kGemmThreads, kGemmSmem, D.sm_count);
  for (int c : kKShares)
    D.gemm_clusters[c] = max_clusters(c, gemm_tc_kernel<EPI_OUT, GEMM_KSPLIT, GEMM_ONE>, kGemmThreads, kGemmSmem, D.sm_count);
  D.gemm_attr = true;
  return LP_OK;
}

// How a product is cut up.
struct GemmCut {
  tc::GemmKind kind;
  int ctas;          // of a cluster
};
static unsigned rows_b(const GemmCut& cut) { return cut.kind == tc::GEMM_HALF ? 64 : 128; }   // of B in a CTA
// Whichever way has its busiest CTA finish first.  A K block of `loads` tiles of 16 KB and `products` of them takes an SM 256
// cycles a load (64 bytes a cycle from L2) or, for each product, 512 cycles (128 x 256 of a pair's tile; 690 with one plane of
// each operand, measured: 0.47 us with 42 pairs at work) or 256 (128 x 128).  Half a pair's tile, 256 x 128, has three products of
// 256 cycles and loads of as many (128 rows of A and 64 of B in two parts, 48 KB): what the last wave leaves idle is halved (fp32
// loss of 1001 x 640 x 20011 in rounds of four K blocks 332 -> 310 us, 2 x 2048 x 512 196 -> 191); with one product a K block its loads would take 1.5 times
// as long as the product.  With few tiles a cluster shares K, at the price of an exchange: about 2500 cycles beside three products
// a K block, 4500 beside one or two, whose K blocks take less than counted here while few SMs draw on L2 (us a call of five steps
// with 800, 2000, 3000, 4500, 6500 cycles: 300 x 400 in fp32 130, 130, 131, 145, 161, 600 x 600 in bf16 126, 126, 126, 115, 116,
// 200 x 200 in bf16 111, 83, 80, 80, 80); 3000 more among eight CTAs, four of which only give their sums away (200 x 8192 in fp32 184 us, 231 on
// clusters of four, in bf16 122 and 131; 64 x 512 x 1000 of the fp32 loss 40.7 and 38.9).
static GemmCut gemm_cut(long long M, long long N, long long K, int batch, bool sym, int a_planes, int b_planes) {
  const Device& D = cur_dev();
  auto count = [&](int t, int u) {
    const long long tm = (M + t - 1) / t, tn = (N + u - 1) / u;
    return (sym ? tm * (tm + 1) / 2 : tm * tn) * batch;
  };
  auto waves = [](long long n, int at_once) { return (n + at_once - 1) / at_once; };
  const int loads = a_planes + b_planes, products = loads - 1;
  const long long kb = (K + 63) / 64, c_pair = std::max(256 * loads, products == 1 ? 690 : 512 * products),
                  c_single = std::max(256 * loads, 256 * products);
  GemmCut best{tc::GEMM_SINGLE, 1};
  long long time = (kb + 2) * c_single * waves(count(128, 128), D.sm_count);
  if (D.gemm_pairs > 0) {
    const long long t = (kb + 2) * c_pair * waves(count(256, 256), D.gemm_pairs);
    if (t <= time) { best = GemmCut{tc::GEMM_PAIR, 2}; time = t; }
    if (products == 3 && !sym) {
      const long long t_half = (kb + 2) * 800 * waves(count(256, 128), D.gemm_pairs);
      if (t_half < time) { best = GemmCut{tc::GEMM_HALF, 2}; time = t_half; }
    }
  }
  for (int c : kKShares) {
    if (c > kb || D.gemm_clusters[c] < 1) continue;
    const long long t = (((kb + c - 1) / c + 2) * c_single + (products == 3 ? 2500 : 4500) + (c == 8 ? 3000 : 0)) * waves(count(128, 128), D.gemm_clusters[c]);
    if (t < time) { best = GemmCut{tc::GEMM_KSPLIT, c}; time = t; }
  }
  return best;
}

template <int kEpi, int kMode>
static cudaError_t start_gemm(const tc::GemmParams& p, const CUtensorMap& ma, const CUtensorMap& mb, const GemmCut& cut, cudaStream_t st) {
  using namespace tc;
  const Device& D = cur_dev();
  const dim3 block(kGemmThreads);
  if (cut.kind == GEMM_PAIR)
    return launch_pdl_cluster(2, gemm_tc_kernel<kEpi, GEMM_PAIR, kMode>, dim3(2 * std::min(p.total_tiles, D.gemm_pairs)), block, kGemmSmem, st,
                              ma, mb, p);
  if constexpr (kMode == GEMM_SPLIT)
    if (cut.kind == GEMM_HALF)
      return launch_pdl_cluster(2, gemm_tc_kernel<kEpi, GEMM_HALF, kMode>, dim3(2 * std::min(p.total_tiles, D.gemm_pairs)), block, kGemmSmem, st,
                                ma, mb, p);
  if (cut.kind == GEMM_KSPLIT)
    return launch_pdl_cluster(cut.ctas, gemm_tc_kernel<kEpi, GEMM_KSPLIT, kMode>, dim3(cut.ctas * p.total_tiles), block, kGemmSmem, st, ma, mb, p);
  return launch_pdl(gemm_tc_kernel<kEpi, GEMM_SINGLE, kMode>, dim3(std::min(p.total_tiles, D.sm_count)), block, kGemmSmem, st, ma, mb, p);
}
// Launches the product.  Sizes, planes and the epilogue's fields of `p` are the caller's; the rest is filled in here.
template <int kEpi>
static int launch_gemm(tc::GemmParams& p, long long K, const CUtensorMap& ma, bool a_mn, const CUtensorMap& mb, bool b_mn, bool bf16,
                       const GemmCut& cut, cudaStream_t st) {
  const bool pair = cut.kind == tc::GEMM_PAIR || cut.kind == tc::GEMM_HALF;
  const int tile_m = pair ? 256 : 128, tile_n = cut.kind == tc::GEMM_PAIR ? 256 : 128;
  p.tiles_m = (p.M + tile_m - 1) / tile_m;
  p.tiles_n = (p.N + tile_n - 1) / tile_n;
  const long long per = p.sym ? (long long)p.tiles_m * (p.tiles_m + 1) / 2 : (long long)p.tiles_m * p.tiles_n;
  if (per * p.batch > (1LL << 30)) return LP_ERR_SIZE;
  p.total_tiles = (int)(per * p.batch);
  p.group_m = std::min(p.tiles_m, pair ? 8 : 16);
  p.kblocks = (int)((K + 63) / 64);
  // K blocks an accumulation: one where fp32 results are wanted; else as many as cost a sum 2^-11 of it (2^14 steps, each cut off by
  // 2^-25 on average)
  if (!p.round_len) p.round_len = p.a_planes == 2 && p.b_planes == 2 ? 1 : 4096;
  p.a_mn = a_mn;
  p.b_mn = b_mn;
  // operand format: bits 7 and 10 (bf16) on top of fp32 accumulation and the shape
  p.idesc = tc::instr_desc_bf16(tile_m, tile_n, a_mn, b_mn) & ~(bf16 ? 0u : ((1u << 7) | (1u << 10)));
  if (kEpi == tc::EPI_OUT) {
    const long long unit = p.out_bf16 ? 16 : 8;
    bool vec = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0 && p.out_ld % unit == 0 && p.N % unit == 0 && p.out_batch % unit == 0;
    if (p.acc) vec = vec && (reinterpret_cast<uintptr_t>(p.acc) & 31) == 0 && p.N % 8 == 0;
    for (int b = 0; p.use_off && b < p.batch; ++b) vec = vec && p.off[b] % unit == 0;
    p.out_vec = vec;
  }
  cudaError_t e;
  if (p.a_planes == 1 && p.b_planes == 1) {
    if (p.kblocks > p.round_len) e = start_gemm<kEpi, tc::GEMM_LONG>(p, ma, mb, cut, st);
    else e = start_gemm<kEpi, tc::GEMM_ONE>(p, ma, mb, cut, st);
  }
  else if (p.a_planes == 2 && p.b_planes == 2) e = start_gemm<kEpi, tc::GEMM_SPLIT>(p, ma, mb, cut, st);
  else if constexpr (kEpi != tc::EPI_CE) e = start_gemm<kEpi, tc::GEMM_LOW>(p, ma, mb, cut, st);
  else return LP_ERR_UNSUPPORTED;
  LP_CUDA_OK(e);
  return LP_OK;
}

}  // namespace lp
