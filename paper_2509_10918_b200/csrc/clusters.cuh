// What a device places of a kernel that is launched in thread-block clusters.
#pragma once

#include "common.cuh"

namespace toma {

// How many clusters of `ctas` CTAs of a kernel the device holds at once (asked once per device; 0: none).
struct ClusterState {
  std::atomic<unsigned long long> raised{0};
  std::atomic<int> known[64];  // per device: 0 unknown, else the answer + 1
};
template <typename Kernel>
int clusters_at_once(Kernel kernel, ClusterState& st, int ctas, int threads, int smem) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (const int k = st.known[dev].load(std::memory_order_relaxed)) return k - 1;
  int clusters = 0;
  bool ok = raise_dynamic_smem(kernel, smem, st.raised) == cudaSuccess;
  if (ok) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ok = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess;
  }
  if (!ok) (void)cudaGetLastError();  // a failed query is an answer, not an error of the caller's stream
  if (!ok || clusters < 0) clusters = 0;
  st.known[dev].store(clusters + 1, std::memory_order_relaxed);
  return clusters;
}

}  // namespace toma
