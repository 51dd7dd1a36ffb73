// What the translation units beside opw_attn.cu need of a stage: a view of its static part, a launch helper, and a
// guard that makes the stage's device current for the length of a call.  Not part of the ABI.
#pragma once
#include <cstdint>

#include <cuda_runtime.h>

#include "opw_attn.h"

struct opw_stage_view {
  int32_t device, num_layers, Hq, Hkv, D, max_batch, max_pages, sms;
  const int32_t* window;        // [num_layers]
  const int64_t* num_pages;     // [num_layers]
  void* const* pool;            // [num_layers]
  uint32_t* status;             // device status word
  int64_t* launches;
  float scale_log2e;
  bool pdl;
};
opw_stage_view opw_view_of(opw_attn_stage_t* stage);

class opw_device_guard {
 public:
  explicit opw_device_guard(int device) : before_(-1), ok_(true) {
    int now = -1;
    if (cudaGetDevice(&now) != cudaSuccess) { (void)cudaGetLastError(); ok_ = false; return; }
    if (now == device) return;
    if (cudaSetDevice(device) != cudaSuccess) { (void)cudaGetLastError(); ok_ = false; return; }
    before_ = now;
  }
  ~opw_device_guard() {
    if (before_ >= 0) (void)cudaSetDevice(before_);
  }
  opw_device_guard(const opw_device_guard&) = delete;
  opw_device_guard& operator=(const opw_device_guard&) = delete;
  bool ok() const { return ok_; }

 private:
  int before_;
  bool ok_;
};

// Do [a, a + an) and [b, b + bn) share a byte?
inline bool opw_overlap(const void* a, size_t an, const void* b, size_t bn) {
  return reinterpret_cast<uintptr_t>(a) < reinterpret_cast<uintptr_t>(b) + bn && reinterpret_cast<uintptr_t>(b) < reinterpret_cast<uintptr_t>(a) + an;
}

// Launch with (or without) programmatic stream serialisation; see launch() in opw_attn.cu.
template <typename... KArgs, typename... Args>
cudaError_t opw_launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, bool pdl, int cluster,
                       Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (pdl) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
