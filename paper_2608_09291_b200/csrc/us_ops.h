// Launching of the kernels that need no handle (internal to the library).
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/unionsparse.h"

namespace us {

// (us_api.cu) The thread's next us_spmm is not behind one whose CTAs take half an SM.
void forget_last_call();

// Launched like the library's other kernels: with programmatic stream serialization; a cluster of `cluster` blocks along x.
cudaError_t ops_launch(const void* kernel, dim3 grid, int block, int64_t smem, cudaStream_t st, void** args, unsigned cluster = 1);
// Allows a kernel up to `most` bytes of dynamic shared memory (the same in every call) and clusters of more than eight, once per device.
cudaError_t ops_kernel_allow(const void* kernel, int most);
// Has a kernel without dynamic shared memory run with as much of it on an SM as there is, once per device: an SM that has to change how it divides its memory first waits
// until it is empty, and so kernels that use much of it would not start beside this one.
cudaError_t ops_kernel_beside(const void* kernel);
// SMs of the current device (148 where there is none).
int ops_sms();
// Address of a __device__ variable on the current device; `kept`: the caller's static array of what was found (by device).
constexpr int kMaxDevices = 64;
cudaError_t ops_symbol(void** kept, const void* symbol, void** address);

}  // namespace us
