// Attention over a latent cache, bf16.
#include "latent_instances.cuh"

template int instinfer::api::launch_latent<__nv_bfloat16>(int32_t, const LatentLaunch &);
