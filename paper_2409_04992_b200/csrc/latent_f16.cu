// Attention over a latent cache, fp16.
#include "latent_instances.cuh"

template int instinfer::api::launch_latent<__half>(int32_t, const LatentLaunch &);
