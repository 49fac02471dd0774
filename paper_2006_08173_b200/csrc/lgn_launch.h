// Launch helper of the operators around the compression path: a kernel that may become resident
// while the kernel before it on the stream is still running (programmatic stream serialisation).
// A kernel launched this way executes griddepcontrol.wait before its first access to global
// memory, which returns when everything before it on the stream has finished and is visible.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "lgn.h"

namespace lgn {

inline lgn_status launch_dependent(const void *fn, dim3 grid, dim3 block, void **args, size_t smem, void *stream,
                                   unsigned cluster = 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    if (cudaLaunchKernelExC(&cfg, fn, args) != cudaSuccess) { (void)cudaGetLastError(); return LGN_ERR_CUDA; }
    return LGN_OK;
}

// SM count of the current device (0: the runtime refused).
inline int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms;
}

inline bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Bytes from the first to the last element of a matrix (rows and cols > 0, ld >= cols), each extent up to 2^40; 0 if they are 2^62 or more,
// which no memory has.
inline uint64_t matrix_bytes(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t es) {
    if ((rows - 1) > ((1ull << 62) / es - cols) / ld) return 0;
    return ((rows - 1) * ld + cols) * es;
}

inline bool ranges_overlap(const void *a, uint64_t an, const void *b, uint64_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return an > 0 && bn > 0 && x < y + bn && y < x + an;
}

}  // namespace lgn

#ifdef __CUDACC__
namespace lgn {
__device__ __forceinline__ void dep_launch() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void dep_wait()   { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Read-only loads that stay behind dep_wait(): the compiler may move a plain load of memory it takes to be
// constant for the kernel's whole run (__ldg, const __restrict__) across it.
__device__ __forceinline__ uint32_t ldro_u32(const void *p) {
    uint32_t v;
    asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t ldro_u64(const void *p) {
    uint64_t v;
    asm volatile("ld.global.nc.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ldro_u16(const void *p) {
    uint16_t v;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
    return v;
}
}  // namespace lgn
#endif
