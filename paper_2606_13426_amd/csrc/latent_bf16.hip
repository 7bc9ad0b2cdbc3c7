// sd_latent_attention's kernels for bf16 queries and caches.
#include "latent.hpp"

namespace sd {
hipError_t latent_bf16_launch(const latent::Args& a, hipStream_t s) { return latent::run_type<latent::Bf16>(a, s); }
}  // namespace sd
