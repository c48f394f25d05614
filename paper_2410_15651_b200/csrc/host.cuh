// Host-side helpers of the entry points: errors, the workspace's layout, argument checks and launches.
#pragma once
#include "../../include/rlhf_ppo.h"

#include <cmath>
#include <cstdint>
#include <cstdio>

#include <cuda_runtime.h>

namespace rlhf {

inline thread_local char g_cuda_error[256] = "";

inline int cuda_fail(cudaError_t e, const char* what)
{
    snprintf(g_cuda_error, sizeof g_cuda_error, "%s: %s", what, cudaGetErrorString(e));
    return RLHF_ERR_CUDA;
}

#define RLHF_CUDA(call)                                   \
    do {                                                  \
        cudaError_t e_ = (call);                          \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call); \
    } while (0)

// Workspace layout (bytes): [0,4) status flags, [4,8) reduction ticket, [8,16) mean and 1/std of the
// advantage whitening, [16,20) row counter of the kernels that deal their rows dynamically, [256, kRowLossOffset) block
// partial sums of the two losses (2 doubles per block of the kernel that reduces them),
// [kRowLossOffset, +4*B*T) per-token policy loss terms (kernels without the fused finalisation), then, for the objectives
// beside step 4, 8*B*T bytes more: per-token KL terms (policy loss with KL); the factor of each sequence and, from
// 4*B*T on, the loss of each pair (preference loss).
constexpr size_t kPartialsOffset = 256;
constexpr size_t kRowLossOffset = 24576;
constexpr int kMaxFusedBlocks = (int)((kRowLossOffset - kPartialsOffset) / 16);   // block partials that fit the header

constexpr long long kMaxTokens = 1ll << 29;
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline int check_shape(int B, int T, int V)
{
    if (B <= 0 || T <= 0 || V <= 0) return RLHF_ERR_SHAPE;
    // the log-prob kernel walks up to 2*B*T rows (two tensors in one launch) plus one grid stride with 32-bit
    // indices, so B*T stays at or below 2^29
    if ((long long)B * (long long)T > kMaxTokens) return RLHF_ERR_SHAPE;
    return RLHF_OK;
}

// Bytes of the workspace that rlhf_ppo_loss_fwd_bwd touches: header + per-token policy loss terms.
inline size_t loss_workspace_bytes(int B, int T) { return kRowLossOffset + 4 * (size_t)B * (size_t)T; }

// Bytes that the other objectives touch.
inline size_t objective_workspace_bytes(int B, int T) { return kRowLossOffset + 12 * (size_t)B * (size_t)T; }

inline int check_workspace(const void* ws, size_t bytes, size_t need)
{
    if (!ws) return RLHF_ERR_NULL;
    if (!aligned(ws, 256)) return RLHF_ERR_ALIGN;
    if (bytes < need) return RLHF_ERR_WORKSPACE;
    return RLHF_OK;
}

struct DeviceInfo {
    int sm_count = 0;
    int max_smem_optin = 0;     // per block
    int smem_per_sm = 0;
};

// Queried per call: the library keeps no state, and the two attributes are cheap to read.
inline int device_info(DeviceInfo& d)
{
    int dev = 0;
    RLHF_CUDA(cudaGetDevice(&dev));
    RLHF_CUDA(cudaDeviceGetAttribute(&d.sm_count, cudaDevAttrMultiProcessorCount, dev));
    RLHF_CUDA(cudaDeviceGetAttribute(&d.max_smem_optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev));
    RLHF_CUDA(cudaDeviceGetAttribute(&d.smem_per_sm, cudaDevAttrMaxSharedMemoryPerMultiprocessor, dev));
    return RLHF_OK;
}

// Launches `kernel` with programmatic stream serialisation allowed (see pdl_wait_prior_grid): the launch
// itself and the kernel's set-up overlap the tail of the kernel before it in the stream.
// `cluster` > 1 launches the grid as thread-block clusters of that many blocks.
inline void fill_launch_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attr)[2], int grid, int block, size_t smem,
                        int cluster, cudaStream_t s)
{
    cfg = cudaLaunchConfig_t{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
}

template <typename... Params, typename... Args>
cudaError_t launch_kernel_cluster(void (*kernel)(Params...), int grid, int block, size_t smem, int cluster,
                                  cudaStream_t s, Args&&... args)
{
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    fill_launch_config(cfg, attr, grid, block, smem, cluster, s);
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

template <typename... Params, typename... Args>
cudaError_t launch_kernel(void (*kernel)(Params...), int grid, int block, size_t smem, cudaStream_t s, Args&&... args)
{
    return launch_kernel_cluster(kernel, grid, block, smem, 1, s, static_cast<Args&&>(args)...);
}

// The row kernels run with the largest shared-memory carve-out.  A kernel that prefers another
// split makes the SMs switch configuration before and after it, which costs microseconds per
// launch; so the small kernels between them ask for the same carve-out.
template <typename K>
int keep_max_carveout(K kernel)
{
    RLHF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    return RLHF_OK;
}

// Temperatures whose square is a number in fp32, and that leave logits of 1e6 below 1e9.  (NaN is none.)
inline bool temperature_ok(float t) { return t >= 1e-3f && t <= 1e18f; }

inline int launch_check(const char* what)
{
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, what);
    return RLHF_OK;
}

}  // namespace rlhf
