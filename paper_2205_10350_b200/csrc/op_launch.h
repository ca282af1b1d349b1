// What the operator-level entry points in more than one source file share (defined in ad_api.cu unless it is a template).
#pragma once

#include <cuda_runtime.h>

#include <utility>

namespace ad {

// Records "entry: why" as the message that ad_last_error(NULL) returns, and returns the code.
int op_fail(int code, const char* entry, const char* why) noexcept;
// The current device (0 .. 63), and its SMs.
int op_device();
int op_num_sms();
// Whether kernels may begin before their predecessor in the stream has ended (they wait for it themselves).
bool op_early_launch();

// Launches a kernel that waits for its predecessor by itself; cluster = dim3() or the number of CTAs along x that form one.
template <typename... KArgs, typename... Args>
cudaError_t launch_op(void (*kernel)(KArgs...), dim3 grid, dim3 block, dim3 cluster, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (op_early_launch()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster.x > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster.x; attr[n].val.clusterDim.y = 1; attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(std::forward<Args>(args))...);
}

}  // namespace ad
