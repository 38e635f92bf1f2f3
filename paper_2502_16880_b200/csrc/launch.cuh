// Host-side checks and launch helpers shared by the translation units of the library.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "coral_lmhead.h"

namespace coral {

// Launch with the programmatic-serialisation attribute: the kernel may begin while the previous kernel of
// the stream is still running and synchronises with it through pdl_wait().
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int elem_size(int type) { return type == CORAL_TYPE_F32 ? 4 : 2; }

inline bool device_sms(int* sms) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess;
}

// The attribute is per kernel and device; above 48 KB, static shared memory (at most kMostStatic in kernels that have both) counted in, it has
// to be raised before the launch.
constexpr size_t kMostStatic = 24 * 1024;
template <typename K>
bool allow_smem(K kernel, size_t bytes) {
    return bytes <= 48 * 1024 - kMostStatic ||
           cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

}  // namespace coral
