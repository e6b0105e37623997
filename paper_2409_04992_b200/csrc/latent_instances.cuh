// The kernels over a latent cache, launched; included by the files that instantiate them.
#pragma once

#include "latent_launch.cuh"

namespace instinfer {
namespace api {

template <typename E, int L, int N>
int launch_latent_instance(const LatentLaunch &t)
{
    using Geo = LatentGeometry<L, N>;
    static bool done[kMaxDevices] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return INSTINFER_ERR_CUDA;
    if (!done[dev]) {
        if (cudaFuncSetAttribute(latent_attn_kernel<E, L, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo::kSmemBytes) != cudaSuccess) {
            (void)cudaGetLastError();
            return INSTINFER_ERR_CUDA;
        }
        done[dev] = true;
    }
    cudaError_t err = launch_overlapped(latent_attn_kernel<E, L, N>, t.grid, Geo::kThreads, Geo::kSmemBytes, t.stream, t.p, t.map_q, t.map_cache);
    if (err != cudaSuccess || cudaGetLastError() != cudaSuccess) return INSTINFER_ERR_CUDA;
    err = launch_overlapped(latent_merge_kernel<E, L>, t.merge_grid, kLatentMergeThreads, 0, t.stream, t.p, t.row_parts);
    return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? INSTINFER_OK : INSTINFER_ERR_CUDA;
}

template <typename E>
int launch_latent(int32_t latent_dim, int32_t columns, const LatentLaunch &t)
{
    if (latent_dim == 512)
        return columns == 16 ? launch_latent_instance<E, 512, 16>(t) : columns == 32 ? launch_latent_instance<E, 512, 32>(t) : launch_latent_instance<E, 512, 64>(t);
    return columns == 16 ? launch_latent_instance<E, 256, 16>(t) : columns == 32 ? launch_latent_instance<E, 256, 32>(t) : launch_latent_instance<E, 256, 64>(t);
}

}  // namespace api
}  // namespace instinfer
