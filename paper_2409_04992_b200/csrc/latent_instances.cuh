// The kernels over a latent cache, launched; included by the files that instantiate them.
#pragma once

#include "latent_launch.cuh"

namespace instinfer {
namespace api {

// Shared-memory opt-in of an instance, once per device.
template <int kSmem, auto kKernel>
int latent_opt_in()
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
    return INSTINFER_OK;
}
template <typename E, int L>
int launch_latent_merge(const LatentLaunch &t, cudaError_t err)
{
    if (err != cudaSuccess || cudaGetLastError() != cudaSuccess) return INSTINFER_ERR_CUDA;
    err = t.merge_dims == L ? launch_overlapped(latent_merge_kernel<E, L, L>, t.merge_grid, kLatentMergeThreads, 0, t.stream, t.p, t.row_parts)
                            : launch_overlapped(latent_merge_kernel<E, L, 128>, t.merge_grid, kLatentMergeThreads, 0, t.stream, t.p, t.row_parts);
    return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? INSTINFER_OK : INSTINFER_ERR_CUDA;
}
template <typename E, int L, int N>
int launch_latent_tokens(const LatentLaunch &t)
{
    using Geo = LatentGeometry<L, N>;
    if (latent_opt_in<Geo::kSmemBytes, latent_attn_kernel<E, L, N>>() != INSTINFER_OK) return INSTINFER_ERR_CUDA;
    return launch_latent_merge<E, L>(t, launch_overlapped(latent_attn_kernel<E, L, N>, t.grid, Geo::kThreads, Geo::kSmemBytes, t.stream, t.p, t.map_q, t.map_cache));
}
template <typename E, int L>
int launch_latent_pairs(const LatentLaunch &t)
{
    using Geo = PairGeometry<L>;
    if (latent_opt_in<Geo::kSmemBytes, latent_pair_kernel<E, L>>() != INSTINFER_OK) return INSTINFER_ERR_CUDA;
    return launch_latent_merge<E, L>(t, launch_clustered(latent_pair_kernel<E, L>, t.grid, 2, kPairThreads, Geo::kSmemBytes, t.stream, t.p, t.map_q, t.map_cache));
}

template <typename E>
int launch_latent(int32_t columns, const LatentLaunch &t)
{
    return columns == 16 ? launch_latent_tokens<E, 512, 16>(t) : columns == 32 ? launch_latent_tokens<E, 512, 32>(t) : launch_latent_pairs<E, 512>(t);
}

}  // namespace api
}  // namespace instinfer
