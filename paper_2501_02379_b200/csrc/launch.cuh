// Host-side launch helpers shared by the translation units of the library.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>

#include "../../include/tgrad.h"

namespace tg {

constexpr int kNoCopyLimit = 0x7fffffff;
extern std::atomic<int> g_copy_limit;     // for tests: copies after which the streaming kernels stop (defined in train_api.cu)
extern std::atomic<int64_t> g_launches;   // kernels launched since the library was loaded (defined in tgrad_api.cu)

#define TG_LAUNCH_CHECK()                                  \
  do {                                                     \
    ::tg::g_launches.fetch_add(1, std::memory_order_relaxed);    \
    if (cudaPeekAtLastError() != cudaSuccess) return TGRAD_ERR_CUDA; \
  } while (0)

// Launch of a kernel with programmatic dependent launch, so that its blocks are scheduled while the previous kernel
// of the stream drains (every such kernel waits, griddep_wait(), before it touches what an earlier one writes).
// cluster > 1: thread-block clusters of that many consecutive blocks.
template <typename... KA, typename... AA>
inline void launch_cluster(void (*kern)(KA...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st, AA&&... args) {
  cudaLaunchConfig_t lc; memset(&lc, 0, sizeof(lc));
  lc.gridDim = grid; lc.blockDim = block; lc.dynamicSmemBytes = smem; lc.stream = st;
  cudaLaunchAttribute at[2]; memset(at, 0, sizeof(at));
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  lc.attrs = at; lc.numAttrs = cluster > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&lc, kern, static_cast<KA>(args)...);     // an error stays pending for TG_LAUNCH_CHECK
}
template <typename... KA, typename... AA>
inline void launch_chained(void (*kern)(KA...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, AA&&... args) {
  launch_cluster(kern, grid, block, smem, 1, st, static_cast<AA&&>(args)...);
}

}  // namespace tg
