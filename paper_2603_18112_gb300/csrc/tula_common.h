// What the library's translation units share on the host.
#pragma once

#include <cuda_runtime.h>

namespace tula {

void note_launch();            // one more of the kernels tula_ags_launch_count counts
void note_cuda_error(int e);   // what tula_ags_last_cuda_error returns on this thread

// Launch with programmatic stream serialization: the kernel may begin while the one before it in
// the stream finishes, and must execute griddepcontrol.wait before it reads or writes anything.
template <typename... KArgs, typename... Args>
int launch(void (*kernel)(KArgs...), dim3 grid, int threads, int smem, cudaStream_t s,
           int cluster, Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
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
    cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Args &&>(args)...);
    note_launch();
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return 0;
    note_cuda_error((int)e);
    return -3;  // TULA_ERR_CUDA
}

}  // namespace tula
