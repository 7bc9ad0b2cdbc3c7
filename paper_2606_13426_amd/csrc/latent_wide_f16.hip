// sd_latent_attention_tree's kernel of 128 rows a workgroup for fp16 queries and caches.
#include "latent_wide.hpp"

namespace sd {
hipError_t latent_wide_f16_launch(const latent::Args& a, hipStream_t s) { return latent::run_wide<latent::F16>(a, s); }
}  // namespace sd
