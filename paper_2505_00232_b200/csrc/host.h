// What the host halves of the library's two translation units share (qlinear.cu: the layers; serving.cu: the operators of a serving step).
#pragma once
#include <cuda_runtime.h>

#include "../../include/qlinear.h"

namespace ql {

// The device's shared state (created on first use), as serving.cu needs it.
struct SharedState {
    int sms = 0;
    volatile unsigned int* status_host = nullptr;    // pinned, mapped: the code of the last expired wait (0 = none)
};
ql_status shared_state(int device, SharedState* out);
ql_status device_sms(int device, int* sms);          // checks the device as well (QL_ERR_ARCH); allocates nothing
bool pdl_enabled();                                  // QLINEAR_PDL
int paged_shared_choice();                           // QLINEAR_PAGED_SHARED
ql_status device_status(int device, uint32_t* detail);   // qlinear_device_status for a device whose shared state exists

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
        if (prev == dev) prev = -1;
    }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

template <typename Kern, typename Params>
cudaError_t launch(Kern kern, const Params& prm, dim3 grid, dim3 block, size_t smem, cudaStream_t st, int cluster, bool pdl)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attrs[2];
    int na = 0;
    if (cluster > 1) {
        attrs[na].id = cudaLaunchAttributeClusterDimension;
        attrs[na].val.clusterDim.x = cluster;
        attrs[na].val.clusterDim.y = 1;
        attrs[na].val.clusterDim.z = 1;
        ++na;
    }
    if (pdl) {
        attrs[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attrs[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    cfg.attrs = attrs;
    cfg.numAttrs = na;
    return cudaLaunchKernelEx(&cfg, kern, prm);
}

}  // namespace ql
