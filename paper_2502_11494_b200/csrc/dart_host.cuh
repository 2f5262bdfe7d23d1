// What the host files of the C ABI share: the device of a call, launches, overlap of two tensors.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace {

// Scoped device switch: the library never leaves another device current.
struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        ok = (prev == dev) || (cudaSetDevice(dev) == cudaSuccess);
        if (prev == dev) prev = -1;
    }
    ~DeviceGuard()
    {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

// Launch behind the kernel before it on the stream, which may still be running (see wait_for_previous): every kernel that is
// launched this way waits before it reads or writes anything that another one touches - but for the gather that follows rank_kernel
// word by word: rank_kernel lets it start behind its own wait, so that all earlier kernels have finished, the words are read and
// published by relaxed accesses at gpu scope and put back behind the gather's wait, which every one of its warps comes to.
// The launch's own result is returned: a kernel that reads indices must not be launched behind one that failed to launch (what a
// launch leaves unnoticed is found by the call's cudaGetLastError).
template <typename... KArgs, typename... Args>
cudaError_t launch_next(void (*kernel)(KArgs...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, Args... args)
{
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
    cfg.attrs = &attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

// Launch behind everything before it on the stream.
template <typename... KArgs, typename... Args>
cudaError_t launch_alone(void (*kernel)(KArgs...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

inline bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    if (!a || !b) return false;
    uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

} // namespace
