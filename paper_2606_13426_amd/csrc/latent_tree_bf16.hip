// sd_latent_attention_tree's kernels for bf16 queries and caches.
#include "latent.hpp"

namespace sd {
hipError_t latent_wide_bf16_launch(const latent::Args& a, hipStream_t s);
hipError_t latent_tree_bf16_launch(const latent::Args& a, hipStream_t s) {
  return a.p.R == latent::kWideR ? latent_wide_bf16_launch(a, s) : latent::run_type<latent::Bf16, true>(a, s);
}
}  // namespace sd
