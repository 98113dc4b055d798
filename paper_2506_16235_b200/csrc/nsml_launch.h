// What the entry points of every source file share: errors of CUDA calls, the kernels' numbers, launches.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "nsml.h"

namespace nsml {

// A CUDA call failed: what the call returns.  The runtime keeps the error of a refused launch or copy for the thread's next
// cudaGetLastError, which is not to meet it again: the calls that follow have nothing to do with it.  (Every launch is
// checked by its own return code.)
inline int cuda_error() {
  cudaGetLastError();
  return NSML_ERR_CUDA;
}

enum KernelId {
  K_SAMPLE = 0, K_COMPACT_BUCKET, K_EMIT, K_PARTITION, K_MERGE, K_CLEAR, K_SELECT_GRID,
  K_SUMSQ, K_PRUNE_PASS, K_PRUNE_FINISH, K_SELECT_SMALL,
  K_Q8_PACK, K_Q8_UNPACK, K_Q8_NORM, K_Q8_NORM_GRAD, K_Q8_NORM_WEIGHT, K_Q8_GEMM, K_Q8_TOKENS, K_COUNT
};

struct LaunchScope {  // brackets one kernel launch
  int id;
  cudaStream_t stream;
  cudaEvent_t start = nullptr, stop = nullptr;
  // timed = false: never bracket this launch with events (creating events allocates)
  LaunchScope(int id_, cudaStream_t s, bool timed = true);
  ~LaunchScope();
};

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int high_priority();  // the device's highest stream priority

// priority: null leaves the stream's
template <class... KArgs, class... Args>
static cudaError_t launch_at(const int* priority, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool cooperative,
                             unsigned int cluster_x, bool dependent, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[4];
  unsigned int na = 0;
  if (priority != nullptr) {
    attr[na].id = cudaLaunchAttributePriority;
    attr[na].val.priority = *priority;
    ++na;
  }
  if (cooperative) {
    attr[na].id = cudaLaunchAttributeCooperative;
    attr[na].val.cooperative = 1;
    ++na;
  }
  if (cluster_x) {
    attr[na].id = cudaLaunchAttributeClusterDimension;
    attr[na].val.clusterDim.x = cluster_x;
    attr[na].val.clusterDim.y = 1;
    attr[na].val.clusterDim.z = 1;
    ++na;
  }
  if (dependent) {  // may start while its predecessor in the stream still runs (programmatic dependent launch); the
                    // kernel calls pdl_wait before it touches anything the predecessor writes
    attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[na].val.programmaticStreamSerializationAllowed = 1;
    ++na;
  }
  cfg.attrs = attr;
  cfg.numAttrs = na;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

// The compression's kernels: a priority of their own, whatever the stream's (high: the device's highest, otherwise 0).
template <class... KArgs, class... Args>
static cudaError_t launch_prio(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool cooperative,
                               unsigned int cluster_x, bool high, bool dependent, Args... args) {
  const int priority = high ? high_priority() : 0;
  return launch_at(&priority, kernel, grid, block, smem, st, cooperative, cluster_x, dependent, args...);
}

// The 8-bit operators' kernels: at the stream's priority, dependent.
template <class... KArgs, class... Args>
static cudaError_t launch_in_stream(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, unsigned int cluster_x, Args... args) {
  return launch_at(nullptr, kernel, grid, block, smem, st, false, cluster_x, true, args...);
}

}  // namespace nsml
