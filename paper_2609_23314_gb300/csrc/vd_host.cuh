// vd_host.cuh -- what the host sides of libvd.so share: the per-device state that
// vd_api.cu owns and the launch of a programmatic dependent kernel.
#pragma once

#include <cuda_runtime.h>

#include "vd.h"
#include "vd_device.cuh"

namespace vd {

struct DeviceInfo {
  int id, sms, smem_optin;
  unsigned* status;  // the device status word
};

// The current device; VD_ERR_NO_DEVICE unless it is an sm_103 one.
vd_status device_info(DeviceInfo* out);

// len[s] += B where the sum stays within cap; a programmatic dependent launch.
vd_status launch_len_add(int32_t* len, int n_seq, int cap, int B, cudaStream_t s);

// What every call on a 4-bit cache checks of it.
vd_status validate_q4(const vd_q4_cache* c);

// Polls after which a device wait gives up (VD_WAIT_LIMIT lowers it, for tests).
uint32_t wait_limit();

// The environment variable's number, or `unset`.
int env_int(const char* name, int unset);

// A plain kernel of `threads`-thread blocks, in clusters of c, as a programmatic
// dependent launch (it waits in griddepcontrol.wait before its first access to memory).
template <class... Params, class... Args>
vd_status launch_clusters(unsigned blocks, unsigned threads, unsigned c, size_t smem,
                          cudaStream_t s, void (*kern)(Params...), Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = c;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = c > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kern, static_cast<Params>(args)...) != cudaSuccess) {
    cudaGetLastError();
    return VD_ERR_CUDA;
  }
  return VD_OK;
}

template <class... Params, class... Args>
vd_status launch_dependent(unsigned blocks, cudaStream_t s, void (*kern)(Params...),
                           Args... args) {
  return launch_clusters(blocks, kThreads, 1, 0, s, kern, args...);
}

}  // namespace vd
