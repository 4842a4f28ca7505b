// Host side shared by the library's translation units: what api.cu keeps per device.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace fsg {

struct DeviceView {
    void*    ws;          // the registered workspace, or nullptr
    uint64_t ws_bytes;
    int      sm_count;
    uint32_t tries;       // of the waits of the losses on logits
    int      device;
};
// The current device's; FASTSGD_OK or FASTSGD_E_CUDA.
int device_view(DeviceView* out);
// Launch bookkeeping (fastsgd_launch_count).
void count_launches(uint64_t launches);
// A launch whose blocks may move onto the GPU while the previous kernel of the stream drains (programmatic dependent launch): the
// kernel itself waits (wait_for_previous_kernels) before it reads or writes memory.  cluster > 1: in clusters of so many blocks.
cudaError_t launch_overlapped(const void* fn, unsigned grid, unsigned threads, size_t smem, void** kargs, cudaStream_t st, unsigned cluster = 1);

}  // namespace fsg
