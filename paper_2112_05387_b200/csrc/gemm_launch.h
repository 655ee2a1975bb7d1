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

// `mn`: the operand's row index is the contiguous one (boxes of 64 rows x 64 K), else K is (128 rows x 64 K).
static int encode_gemm_map(CUtensorMap* m, const GemmOperand& o, bool mn) {
  cuuint64_t dims[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)o.count};
  cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.stride * 2};
  cuuint32_t box[3] = {64, mn ? 64u : 128u, 1};
  cuuint32_t es[3] = {1, 1, 1};
  CUresult r = cur_dev().encode(m, o.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                            const_cast<void*>(o.p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? LP_OK : LP_ERR_CUDA;
}

template <int kEpi>
static int gemm_set_attributes(Device& D) {
  LP_CUDA_OK(cudaFuncSetAttribute(tc::gemm_tc_kernel<kEpi, true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc::kGemmSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(tc::gemm_tc_kernel<kEpi, false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc::kGemmSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(tc::gemm_tc_kernel<kEpi, true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc::kGemmSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(tc::gemm_tc_kernel<kEpi, false, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc::kGemmSmem));
  return LP_OK;
}
// Kernel attributes, and how many CTA pairs the device holds at once (the grid is persistent: never more than that).
static int gemm_init_dev() {
  int rc = init_cur_dev();
  if (rc != LP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_devices_mutex);
  Device& D = cur_dev();
  if (D.gemm_attr) return LP_OK;
  if ((rc = gemm_set_attributes<tc::EPI_H16>(D)) != LP_OK) return rc;
  if ((rc = gemm_set_attributes<tc::EPI_OUT>(D)) != LP_OK) return rc;
  if ((rc = gemm_set_attributes<tc::EPI_CE>(D)) != LP_OK) return rc;
  cudaLaunchConfig_t q = {};
  q.gridDim = dim3(2 * D.sm_count);
  q.blockDim = dim3(tc::kGemmThreads);
  q.dynamicSmemBytes = tc::kGemmSmem;
  cudaLaunchAttribute qa[1];
  qa[0].id = cudaLaunchAttributeClusterDimension;
  qa[0].val.clusterDim.x = 2; qa[0].val.clusterDim.y = 1; qa[0].val.clusterDim.z = 1;
  q.attrs = qa;
  q.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, tc::gemm_tc_kernel<tc::EPI_OUT, true, false>, &q) != cudaSuccess) { cudaGetLastError(); n = 0; }
  D.gemm_pairs = n;
  D.gemm_attr = true;
  return LP_OK;
}

// Tiles of 256 x 256 on CTA pairs, or of 128 x 128 on single CTAs: whichever has the busiest CTA finish first.  A pair's tile
// is two of the others' work for each of its CTAs and fetches half as much per product.
static bool gemm_pair_tiles(long long M, long long N, int batch, bool sym, int sms, int pairs) {
  if (pairs < 1) return false;
  auto count = [&](int t) {
    const long long tm = (M + t - 1) / t, tn = (N + t - 1) / t;
    return (sym ? tm * (tm + 1) / 2 : tm * tn) * batch;
  };
  const double pair = 2.0 * ((count(256) + pairs - 1) / pairs), single = 1.3 * ((count(128) + sms - 1) / sms);
  return pair <= single;
}

// K steps (of 64 wide blocks and segments) that the tensor core adds up before its accumulator is emptied into registers
// where fp32 results are wanted.
constexpr int kGemmRound = 12;

// Launches the product.  Sizes, segments and the epilogue's fields of `p` are the caller's; the rest is filled in here.
template <int kEpi>
static int launch_gemm(tc::GemmParams& p, long long K, const CUtensorMap& ma, bool a_mn, const CUtensorMap& mb, bool b_mn, bool bf16,
                       bool rounds, bool pair, cudaStream_t st) {
  const Device& D = cur_dev();
  const int tile = pair ? 256 : 128;
  p.tiles_m = (p.M + tile - 1) / tile;
  p.tiles_n = (p.N + tile - 1) / tile;
  const long long per = p.sym ? (long long)p.tiles_m * (p.tiles_m + 1) / 2 : (long long)p.tiles_m * p.tiles_n;
  if (per * p.batch > (1LL << 30)) return LP_ERR_SIZE;
  p.total_tiles = (int)(per * p.batch);
  p.group_m = std::min(p.tiles_m, pair ? 8 : 16);
  p.kblocks = (int)((K + 63) / 64);
  p.round_len = kGemmRound;
  p.a_mn = a_mn;
  p.b_mn = b_mn;
  // operand format: bits 7 and 10 (bf16) on top of fp32 accumulation and the shape
  p.idesc = tc::instr_desc_bf16(tile, tile, a_mn, b_mn) & ~(bf16 ? 0u : ((1u << 7) | (1u << 10)));
  const dim3 block(tc::kGemmThreads);
  cudaError_t e;
  if (pair) {
    const dim3 grid(2 * std::min(p.total_tiles, D.gemm_pairs));
    e = rounds ? launch_pdl_pair(tc::gemm_tc_kernel<kEpi, true, true>, grid, block, tc::kGemmSmem, st, ma, mb, p)
               : launch_pdl_pair(tc::gemm_tc_kernel<kEpi, true, false>, grid, block, tc::kGemmSmem, st, ma, mb, p);
  } else {
    const dim3 grid(std::min(p.total_tiles, D.sm_count));
    e = rounds ? launch_pdl(tc::gemm_tc_kernel<kEpi, false, true>, grid, block, tc::kGemmSmem, st, ma, mb, p)
               : launch_pdl(tc::gemm_tc_kernel<kEpi, false, false>, grid, block, tc::kGemmSmem, st, ma, mb, p);
  }
  LP_CUDA_OK(e);
  return LP_OK;
}

}  // namespace lp
