// op_launch.cuh -- what the entry points of the sequence-policy operators (linattn.cu, group_norm.cu,
// policy_loss.cu) share on the host: checks of addresses and the launch of a kernel that may start
// while the one before it in the stream drains (see tc::after_previous()).
#pragma once
#include <stdint.h>

#include "kernels.h"
#include "tc_common.cuh"

namespace aht {

aht_status set_last_error(aht_status s, const char* msg);  // the message of aht_last_error

inline aht_status launched(cudaError_t e) {
  return e == cudaSuccess ? AHT_OK : set_last_error(AHT_ECUDA, cudaGetErrorString(e));
}

constexpr char kMisalignedArray[] = "an array is not on a boundary of its elements' size";

// Whether every address is a multiple of `bytes` (NULL is one).
template <typename... P>
bool on_boundary(int bytes, const P*... p) {
  return (((uintptr_t)p % bytes == 0) && ...);
}

// Grid, block, dynamic shared memory and CTAs of a cluster of a launch; `most`: the most that any launch of the kernel has.
// (A kernel's limit belongs to the device, not to a call: every call that sets it sets the same one, or a call of another
// thread could lower it between this one's setting and its launch.)
struct Shape {
  dim3 grid, block;
  int smem = 0, cluster = 1, most = smem;
};

template <typename K, typename... Args>
aht_status launch_op(K kernel, const Shape& sh, cudaStream_t s, const Args&... args) {
  if (sh.smem > 16 * 1024)  // (with the static part it may pass 48 KB)
    if (aht_status e = launched(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sh.most))) return e;
  if (sh.cluster > 8)  // beyond what every device runs
    if (aht_status e = launched(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = sh.grid;
  cfg.blockDim = sh.block;
  cfg.dynamicSmemBytes = (size_t)sh.smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)sh.cluster, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = sh.cluster > 1 ? 2 : 1;
  return launched(cudaLaunchKernelEx(&cfg, kernel, args...));
}

}  // namespace aht
