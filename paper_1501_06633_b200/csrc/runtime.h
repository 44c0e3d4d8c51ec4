// What the translation units of the library share of its per-device state: the device check,
// the status block that kernels report into, tensor-copy descriptors and the launch counter.
#pragma once
#include <atomic>

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/maxdnn.h"
#include "ptx_util.cuh"

namespace maxdnn {

struct RuntimeDevice {
  void* state;      // the DeviceState it was read from
  int index;        // the current device
  int sm_count;
};

// The current device, set up on first use (not during stream capture); NOT_SUPPORTED where it
// is not sm_100.
maxdnn_status runtime_device(RuntimeDevice* out);

// Status block and number of one launch on that device.
WaitCtx runtime_wait_ctx(const RuntimeDevice& dev);

// dims[0] is the contiguous dimension; strides[i] is the byte pitch of dims[i+1].
maxdnn_status runtime_encode(CUtensorMap* m, CUtensorMapDataType dt, int rank, const void* base,
                             const uint64_t* dims, const uint64_t* strides, const uint32_t* box,
                             CUtensorMapSwizzle swz);

void runtime_count_launch();

}  // namespace maxdnn
