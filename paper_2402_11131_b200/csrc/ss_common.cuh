// Internal helpers shared by the CUDA translation units of libss_msa.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>
#include <algorithm>

#include "ss_msa.h"

namespace ss {

// Workspace header: word 0 = device status, the rest of the first 256 bytes is reserved.
constexpr size_t kWsHeaderBytes = 256;

__device__ __forceinline__ void set_status(void* workspace, int32_t code) {
    atomicCAS(reinterpret_cast<int*>(workspace), 0, code);   // keep the first error
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int sm_count() {
    static int cached[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    if (cached[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
        cached[dev] = n;
    }
    return cached[dev];
}

// A cache in 4 bits: what the host can see of it.
inline int32_t kvq_check_cache(const ss_kvq_cache& c) {
    if (!c.k_codes || !c.v_codes || !c.k_params || !c.v_params || c.n_layers < 1 || c.n_heads < 1 || c.total_slots < 0 || c.total_slots > 1ll << 48) return SS_ERR_INVALID_ARG;
    if ((c.head_dim != 64 && c.head_dim != 80 && c.head_dim != 128) || c.n_heads > 65535) return SS_ERR_UNSUPPORTED;
    const uintptr_t unit = c.head_dim == 80 ? 7u : 15u;
    if (((reinterpret_cast<uintptr_t>(c.k_codes) | reinterpret_cast<uintptr_t>(c.v_codes)) & unit) ||
        ((reinterpret_cast<uintptr_t>(c.k_params) | reinterpret_cast<uintptr_t>(c.v_params)) & 3u))
        return SS_ERR_INVALID_ARG;
    if (static_cast<uintptr_t>(c.layer_stride | c.slot_stride | c.head_stride) & unit) return SS_ERR_UNSUPPORTED;
    if (c.device < -1) return SS_ERR_INVALID_ARG;
    int dev = -1;
    if (c.device >= 0 && (cudaGetDevice(&dev) != cudaSuccess || dev != c.device)) return SS_ERR_INVALID_ARG;
    return SS_OK;
}

// Programmatic dependent launch.  A kernel launched with launch_after_previous may be scheduled while the
// previous kernel of the stream drains; it must call wait_for_previous_kernel() before it touches global
// memory, which restores plain stream order for everything after the call.
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The other half: lets the next kernel of the stream be scheduled from here on.  Called after the wait only, so at most
// two kernels of a stream are ever on the GPU: what ran before the previous kernel is complete.  A kernel that writes tree
// descriptors calls it only once they are in memory, or not at all: an attention call behind it may promise that they are
// stable and reads them before its wait.
__device__ __forceinline__ void release_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// `cluster` CTAs along x form a cluster; early: may be scheduled while the previous kernel of the stream drains
template <typename... KArgs, typename... Args>
inline cudaError_t launch_rows(void (*kernel)(KArgs...), dim3 grid, dim3 block, int cluster, bool early, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (early) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = static_cast<unsigned>(cluster);
        attr[n].val.clusterDim.y = 1;
        attr[n++].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = static_cast<unsigned>(n);
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

template <typename... KArgs, typename... Args>
inline cudaError_t launch_after_previous(void (*kernel)(KArgs...), dim3 grid, dim3 block, cudaStream_t stream, Args... args) {
    return launch_rows(kernel, grid, block, 1, true, stream, args...);
}

}  // namespace ss
