// sd_latent_attention_tree's kernel of 128 rows a workgroup for bf16 queries and caches.
#include "latent_wide.hpp"

namespace sd {
hipError_t latent_wide_bf16_launch(const latent::Args& a, hipStream_t s) { return latent::run_wide<latent::Bf16>(a, s); }
}  // namespace sd
