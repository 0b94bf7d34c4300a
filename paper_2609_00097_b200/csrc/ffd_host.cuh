// Host helpers that the sources of the library share: argument checks, launches, sizes.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/ffd.h"
#include "ffd_kernels.cuh"

namespace ffd {

constexpr size_t kHeaderBytes = 256;
// ffd_workspace_init does not know the geometry: it zeroes the header and as many arrival counters as any geometry can
// have (one per (sequence, KV head), fewer than 65536 of them)
constexpr size_t kInitBytes = kHeaderBytes + 65536 * sizeof(uint32_t);

static inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// SM count of the current device; 148 (B200) when no device can be asked, so that the host-only entry points still
// answer.  Asked on every call: the library caches nothing, and the answer must follow cudaSetDevice.
constexpr int kDefaultSms = 148;
static inline int device_sms() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) {
        (void)cudaGetLastError();
        return kDefaultSms;
    }
    return sms;
}

static inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

static inline ffd_status check_geometry(int batch, int max_blocks, int num_pages) {
    if (batch <= 0 || batch > 65535 || max_blocks <= 0 || num_pages <= 0) return FFD_ERR_SHAPE;
    if ((long)max_blocks * kBlk > 0x7fffffffL) return FFD_ERR_SHAPE;
    return FFD_OK;
}

// Launch with programmatic stream serialization: the grid may be scheduled while its predecessor in the stream is
// still running; every kernel of this library calls pdl_wait() before it reads anything a predecessor wrote.
template <typename... KArgs, typename... Args>
static inline void launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    (void)cudaLaunchKernelEx(&cfg, kernel, args...);   // errors surface through cudaGetLastError in launch_status
}

static inline ffd_status launch_status() { return cudaGetLastError() == cudaSuccess ? FFD_OK : FFD_ERR_CUDA; }

}  // namespace ffd
