// Host side shared by the library's translation units: what api.cu keeps per device.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

#include "../../include/fastsgd.h"

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

// ---- checks and launches of the calls on matrices -------------------------------------------------
inline uint32_t size_of(uint32_t type) { return type == FASTSGD_F32 ? 4u : 2u; }
inline bool is_type(uint32_t type) { return type == FASTSGD_F32 || type == FASTSGD_BF16 || type == FASTSGD_F16; }
inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int check_matrix(const fastsgd_matrix* m) {
    if (!m) return FASTSGD_E_NULL;
    if (!is_type(m->type) || m->reserved) return FASTSGD_E_BAD_PARAM;
    if (m->rows >= (1ull << 31) || m->cols == 0 || m->cols >= (1ull << 31)) return FASTSGD_E_BAD_N;
    if (m->row_stride < m->cols || m->row_stride >= (1ull << 31)) return FASTSGD_E_BAD_PARAM;
    if (m->rows && !m->data) return FASTSGD_E_NULL;
    if (!aligned_to(m->data, size_of(m->type))) return FASTSGD_E_ALIGN;
    return FASTSGD_OK;
}

inline uint64_t span_bytes(const fastsgd_matrix* m) { return m->rows ? ((m->rows - 1) * m->row_stride + m->cols) * size_of(m->type) : 0; }

inline int launched(cudaError_t err, uint64_t launches = 1) {
    if (err != cudaSuccess) { cudaGetLastError(); return FASTSGD_E_CUDA; }
    count_launches(launches);
    return FASTSGD_OK;
}

// Blocks of a kernel that stay on the GPU at once; it may then use as much shared memory, and run in clusters of sixteen blocks (asked for once per device, kernel and size; asking costs as much as a small launch).
struct Residency { int dev; const void* fn; size_t smem; uint64_t blocks; };
constexpr int kResidencies = 256;
inline std::mutex g_residency_mu;
inline Residency g_residency[kResidencies];
inline int g_residencies = 0;
inline int resident_blocks(const void* fn, int threads, size_t smem, const DeviceView& dev, uint64_t* out) {
    std::lock_guard<std::mutex> lock(g_residency_mu);
    for (int i = 0; i < g_residencies; ++i) {
        const Residency& r = g_residency[i];
        if (r.fn == fn && r.smem == smem && r.dev == dev.device) { *out = r.blocks; return FASTSGD_OK; }
    }
    int per_sm = 0, most = 0;
    cudaFuncAttributes at;
    if (cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev.device) != cudaSuccess || cudaFuncGetAttributes(&at, fn) != cudaSuccess
        || cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, most - (int)at.sharedSizeBytes) != cudaSuccess
        || cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        cudaGetLastError();
        return FASTSGD_E_CUDA;
    }
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, fn, threads, smem) != cudaSuccess || per_sm < 1) { cudaGetLastError(); return FASTSGD_E_CUDA; }
    *out = (uint64_t)per_sm * (uint64_t)dev.sm_count;
    g_residency[g_residencies < kResidencies ? g_residencies++ : kResidencies - 1] = Residency{dev.device, fn, smem, *out};
    return FASTSGD_OK;
}

}  // namespace fsg
