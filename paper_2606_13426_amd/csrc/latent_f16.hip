// sd_latent_attention's kernels for fp16 queries and caches, and the choice of type and form.
#include "latent.hpp"

namespace sd {

hipError_t latent_bf16_launch(const latent::Args& a, hipStream_t s);
hipError_t latent_tree_bf16_launch(const latent::Args& a, hipStream_t s);
hipError_t latent_tree_f16_launch(const latent::Args& a, hipStream_t s);

namespace {
inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int padded(int dc) { return (dc + 127) / 128 * 128; }
struct Layout {
  size_t part, stat, first, last, bytes;
};
Layout layout(int B, int dc, const latent::Plan& p) {
  const size_t rows = (size_t)latent::kGroups * 2 * 16 * p.R;
  Layout l;
  l.part = 0;
  l.stat = up256(rows * padded(dc) * sizeof(float));
  l.first = l.stat + up256(rows * sizeof(float2));
  l.last = l.first + up256((size_t)B * p.supers * sizeof(int32_t));
  l.bytes = l.last + up256((size_t)B * p.supers * sizeof(int32_t));
  return l;
}
}  // namespace

// Enough for pages of any size (the smallest give the fewest rows a workgroup).
size_t latent_ws_bytes(int B, int Q, int H, int dc) {
  const int64_t rows = (int64_t)Q * H;
  size_t most = 0;
  for (int R = latent::most_r(rows); R >= latent::plan(B, Q, H, 1).R; R /= 2) {
    const size_t bytes = layout(B, dc, latent::plan_of(rows, R)).bytes;
    most = bytes > most ? bytes : most;
  }
  return most;
}
size_t latent_tree_ws_bytes(int B, int Q, int H, int dc, int dr) {
  const size_t few = latent_ws_bytes(B, Q, H, dc);
  if (!latent::wide_fits((int64_t)Q * H, dc, dr)) return few;
  const size_t wide = layout(B, dc, latent::plan_of((int64_t)Q * H, latent::kWideR)).bytes;
  return few > wide ? few : wide;
}

static latent::Args args_of(int B, int Q, int H, int dc, int dr, double scale, const void* q, sd_stride_h qs,
                            const void* cache, int64_t page_stride, int64_t token_stride, int n_pages, int page_size,
                            const int32_t* pages, int64_t pages_stride, int max_pages, const int32_t* lens,
                            const int32_t* rows, const int32_t* parents, void* out, sd_stride_h os, float* lse,
                            void* ws) {
  // (parents: the tree form)
  latent::Args a;
  a.B = B;
  a.Q = Q;
  a.H = H;
  a.dc = dc;
  a.dr = dr;
  // |scale| at least 1e-30, so that a masked score stays -inf where scale is 0
  a.c = (float)fmax(fabs(scale) * 1.44269504088896340736, 1e-30);
  a.flip = scale < 0.0 ? 0x80008000u : 0u;
  a.q = static_cast<const uint16_t*>(q);
  a.qs = qs.seq;
  a.qr = qs.row;
  a.qh = qs.head;
  a.cache = static_cast<const uint16_t*>(cache);
  a.page_stride = page_stride;
  a.token_stride = token_stride;
  a.n_pages = n_pages;
  a.page_size = page_size;
  a.pages = pages;
  a.pages_stride = pages_stride;
  a.capacity = pages ? max_pages * page_size : page_size;
  a.lens = lens;
  a.rows = rows;
  a.parents = parents;
  a.out = static_cast<uint16_t*>(out);
  a.os = os.seq;
  a.orow = os.row;
  a.oh = os.head;
  a.lse = lse;
  a.p = parents ? latent::tree_plan(B, Q, H, dc, dr, a.capacity) : latent::plan(B, Q, H, a.capacity);
  const Layout l = layout(B, dc, a.p);
  char* base = static_cast<char*>(ws);
  a.part = reinterpret_cast<float*>(base + l.part);
  a.stat = reinterpret_cast<float2*>(base + l.stat);
  a.first = reinterpret_cast<int32_t*>(base + l.first);
  a.last = reinterpret_cast<int32_t*>(base + l.last);
  return a;
}

hipError_t latent_launch(int B, int Q, int H, int dc, int dr, sd_type type, double scale, const void* q, sd_stride_h qs,
                         const void* cache, int64_t page_stride, int64_t token_stride, int n_pages, int page_size,
                         const int32_t* pages, int64_t pages_stride, int max_pages, const int32_t* lens,
                         const int32_t* rows, void* out, sd_stride_h os, float* lse, void* ws, hipStream_t s) {
  const latent::Args a = args_of(B, Q, H, dc, dr, scale, q, qs, cache, page_stride, token_stride, n_pages, page_size, pages,
                                 pages_stride, max_pages, lens, rows, nullptr, out, os, lse, ws);
  return type == SD_TYPE_BF16 ? latent_bf16_launch(a, s) : latent::run_type<latent::F16>(a, s);
}

hipError_t latent_tree_launch(int B, int Q, int H, int dc, int dr, sd_type type, double scale, const void* q, sd_stride_h qs,
                              const void* cache, int64_t page_stride, int64_t token_stride, int n_pages, int page_size,
                              const int32_t* pages, int64_t pages_stride, int max_pages, const int32_t* lens,
                              const int32_t* rows, const int32_t* parents, void* out, sd_stride_h os, float* lse,
                              void* ws, hipStream_t s) {
  const latent::Args a = args_of(B, Q, H, dc, dr, scale, q, qs, cache, page_stride, token_stride, n_pages, page_size, pages,
                                 pages_stride, max_pages, lens, rows, parents, out, os, lse, ws);
  return type == SD_TYPE_BF16 ? latent_tree_bf16_launch(a, s) : latent_tree_f16_launch(a, s);
}

}  // namespace sd
