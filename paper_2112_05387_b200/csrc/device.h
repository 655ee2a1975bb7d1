// What every translation unit of the library needs on the host: the record of a device (SM count, tensor-map encoder, kernel
// attributes set so far), error and size helpers, launches on clusters.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <mutex>
#include <utility>

#include "../../include/lp.h"
#include "common.cuh"

namespace lp {

#define LP_CUDA_OK(expr)                         \
  do {                                           \
    cudaError_t e__ = (expr);                    \
    if (e__ != cudaSuccess) return LP_ERR_CUDA;  \
  } while (0)

static inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
static inline size_t esize(int dtype) { return dtype == LP_F32 ? 4 : 2; }

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct Device {
  bool ready = false;
  int sm_count = 148;
  EncodeTiledFn encode = nullptr;
  // kernel attributes are per device: set on the first launch of each kernel family on that device
  bool conv_attr = false, wgrad_attr = false, wgrad_halo_attr = false, conv2_attr = false, f32_attr = false, thin_attr = false,
       gemm_attr = false, ortho_attr = false, ce_attr = false;
  int max_pairs = 0;   // CTA pairs of conv_tc2_kernel that can be resident at once (0: not usable)
  int gemm_pairs = 0;  // the same for gemm_tc_kernel
  int small_clusters[9] = {0}; // clusters of 1, 2, 4, 8 CTAs of ortho_small_kernel
  int gemm_clusters[9] = {0};  // and its clusters of kKShares CTAs (gemm_launch.h) that share K
  int init() {
    if (ready) return LP_OK;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return LP_ERR_CUDA;
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, dev) != cudaSuccess) return LP_ERR_CUDA;
    sm_count = prop.multiProcessorCount;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || !fn)
      return LP_ERR_CUDA;
    encode = (EncodeTiledFn)fn;
    if (prop.major != 10) return LP_ERR_UNSUPPORTED;  // the kernels are built for sm_100a only
    ready = true;
    return LP_OK;
  }
};
// One record per device ordinal; the current device's record is looked up at every use.  The mutex
// covers first-use initialisation from several host threads.
constexpr int kMaxDevices = 64;
inline Device g_devices[kMaxDevices];
inline std::mutex g_devices_mutex;
inline Device& cur_dev() {
  int d = 0;
  if (cudaGetDevice(&d) != cudaSuccess || d < 0 || d >= kMaxDevices) d = 0;
  return g_devices[d];
}
inline int init_cur_dev() {
  std::lock_guard<std::mutex> lock(g_devices_mutex);
  return cur_dev().init();
}

static inline int grid_for(long long work_items, int threads, int sm_count, int per_sm = 8) {
  long long blocks = (work_items + threads - 1) / threads;
  long long cap = (long long)sm_count * per_sm;
  if (blocks > cap) blocks = cap;
  if (blocks < 1) blocks = 1;
  return (int)blocks;
}

// Launch with clusters of `ctas` CTAs and programmatic stream serialisation allowed.
template <typename... KArgs, typename... Args>
static inline cudaError_t launch_pdl_cluster(int ctas, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                                             Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = LP_PDL;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ctas;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
template <typename... KArgs, typename... Args>
static inline cudaError_t launch_pdl_pair(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  return launch_pdl_cluster(2, kernel, grid, block, smem, st, std::forward<Args>(args)...);
}

}  // namespace lp
