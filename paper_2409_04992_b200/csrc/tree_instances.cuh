// The tcgen05 kernels for draft trees, launched; included by the files that instantiate them.
#pragma once

#include "tree_launch.cuh"
#include "tree_umma_rows.cuh"
#include "tree_umma_tokens.cuh"

namespace instinfer {
namespace api {

// `kernel` and the merge behind it; kSmem and the kernel's address are the instance's own.
template <int D, int kSmem, int kThreadsOf, auto kKernel>
int launch_tree_umma(const TreeLaunch &t)
{
    static bool done[kMaxDevices] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return INSTINFER_ERR_CUDA;
    if (!done[dev]) {
        if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return INSTINFER_ERR_CUDA;
        }
        done[dev] = true;
    }
    if (t.draws && cudaMemsetAsync(t.p.ticket, 0, sizeof(unsigned), t.stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return INSTINFER_ERR_CUDA;
    }
    cudaError_t err = launch_overlapped(kKernel, t.grid, kThreadsOf, kSmem, t.stream, t.p, t.map_q, t.map_k, t.map_v);
    if (err != cudaSuccess || cudaGetLastError() != cudaSuccess) return INSTINFER_ERR_CUDA;
    err = launch_overlapped(tree_merge_kernel<D>, t.merge_grid, kTreeMergeThreads, 0, t.stream, t.p, t.row_parts);
    return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? INSTINFER_OK : INSTINFER_ERR_CUDA;
}
template <int D, bool kPaged, int kStreams>
int launch_tree_rows(const TreeLaunch &t)
{
    using Geo = TreeRowsGeometry<D, kStreams>;
    return launch_tree_umma<D, Geo::kSmemBytes, Geo::kThreads, tree_attn_rows_kernel<D, kPaged, kStreams>>(t);
}
template <int D, bool kPaged, int N>
int launch_tree_tokens(const TreeLaunch &t)
{
    return launch_tree_umma<D, TreeTokensGeometry<D, N>::kSmemBytes, TreeTokensGeometry<D, N>::kThreads, tree_attn_tokens_kernel<D, kPaged, N>>(t);
}
template <int D, bool kPaged>
int launch_tree(const TreeRows &rows, const TreeLaunch &t)
{
    if constexpr (D != 64) {                       // (head size 64: the warp-level form)
        if (rows.columns == 16) return launch_tree_tokens<D, kPaged, 16>(t);
    }
    if (rows.columns == 32) return launch_tree_tokens<D, kPaged, 32>(t);
    if (rows.columns == 64) return launch_tree_tokens<D, kPaged, 64>(t);
    if constexpr (D != 256) {
        if (rows.streams == 2) return launch_tree_rows<D, kPaged, 2>(t);
    }
    return launch_tree_rows<D, kPaged, 1>(t);
}

}  // namespace api
}  // namespace instinfer
