// How the host side launches a kernel.
#pragma once
#include <cuda_runtime.h>
#include <string.h>

#include "../../include/mtpc.h"

namespace mtpc {

inline int check_launch() { return cudaGetLastError() == cudaSuccess ? MTPC_OK : MTPC_ERR_CUDA; }

// Launch `kernel`, optionally allowed to start before the kernel ahead of it in the stream has finished (programmatic
// dependent launch): such a kernel calls grid_dependency_wait() before it touches global memory, so what overlaps is its launch and
// set-up (about 2 us a kernel). cluster > 1: in clusters of that many CTAs.
// Five kernels do more before they wait. A kernel that lets its dependents in after its own wait (a gate) has nothing unfinished ahead of
// it, so whatever was launched before it has ended when anything behind it starts; each of the five relies on one:
//   draft_slot_kernel, circuit_hmm_kernel and the static HMM's Eq. 6 kernel copy the head's static tables. The tables are written by a plain
//     launch (bind_parameters), and the first kernel of every call that runs one of the three is a gate (the fp32 conversion, the projection,
//     the weight pass; an acceptance call, whose first kernel may be circuit_hmm_kernel, needs a draft since the last update).
//   loss_coeff_kernel reads the targets and writes the coefficients. The projection it is launched behind is a gate (on a factored head the
//     merge), so the caller's writes and the readers of the last call's coefficients are done.
//   loss_partial_kernel, beside the last GEMM, reads the prefixes and writes its partial sums. The GEMMs are NOT gates, they let their
//     dependents in before they wait. What lies between them and the circuit is: logit_gradient_kernel, by its plain launch, or on a factored
//     head lowrank_pad_kernel. Whoever makes the one a dependent or lets the other's dependents in early breaks the loss.
template <typename... Params, typename... Args>
void launch_clusters(void (*kernel)(Params...), int cluster, dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool dependent,
                     Args&&... args) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (dependent) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
template <typename... Params, typename... Args>
void launch_kernel(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool dependent, Args&&... args) {
  launch_clusters(kernel, 1, grid, block, smem, st, dependent, args...);
}

}  // namespace mtpc
