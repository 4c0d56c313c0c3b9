// cg_follow.cuh -- launches that come while the stream's last kernel ends: the kernel's CTAs are on their SMs, and what
// needs no memory of others is done, when the last one's results are there (programmatic launch). In a row of the
// same call that the host is ahead of, with and without: a plan 1.6 us and 4.1, a commit 4.0 and 6.2, an encoding of 8192 x 4096 (half
// of it in L2) 16.8 and 19.1, a product of one row 6.4 and 8.2, of 333 8.6 and 11.2, the attention of one small tree 15.5 and 17.9; in a
// graph a plan 1.6 and 1.9, a commit 4.0 both ways, the products 6.4 and 6.8, 8.4 and 9.0. CTAs that wait here hold their place on the
// SM: behind a paged attention of few rows, which lets the next kernel come from its first instruction on, both calls together take
// 1 % less (16 requests after 4096 tokens, then a product of one row: 65.5 us and 66.2) to 1 % more (then a product of 2048 rows:
// 112.1 and 110.8; 64 requests after 8192 tokens, then an encoding of 64 rows: 327.6 and 325.7).
#pragma once

#include <cuda_runtime.h>

namespace cg {

// Behind this a kernel of launch_following may read and write what kernels before it wrote and read. Each thread that
// does so calls it first. Loads behind it are ordinary ones: the compiler may move those by way of the read-only path
// (__ldg) before it.
__device__ __forceinline__ void follow() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The next such kernel may come as soon as all CTAs of this one have started, to where they leave room. For kernels of a CTA an SM
// (17 x 6144 x 4096 9.1 us with it and 9.6 without); where several share an SM the next kernel's crowd where this one's end
// first (a product of one row, 4096 x 14336: 16.5 and 12.1).
__device__ __forceinline__ void let_follow() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// cluster: CTAs of a cluster (0: as the kernel says).
template <class... Params, class... Args>
cudaError_t launch_following(void (*kernel)(Params...), unsigned grid, int threads, size_t smem, cudaStream_t st, int cluster, const Args&... args) {
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace cg
