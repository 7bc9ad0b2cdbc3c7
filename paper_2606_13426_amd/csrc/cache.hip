// What writes a paged latent cache: new tokens' vectors with the position rotation on
// the way, and the move of an accepted branch's vectors (gfx950).
//
// Append.  A wavefront takes one token and one part of it: part 0 its cached vector, 16
// bytes a lane, each later part up to 4 heads a lane of the queries' rotary parts, four
// pairs a lane.  A lane's four angles are pos freq in float64, reduced to [-pi/4, pi/4]
// there, with sine and cosine by their power series in float32 (the first terms left out,
// r^11 / 11! and r^12 / 12!, are below 2^-29); its heads share them.
//
// Keep.  A wavefront takes one sequence in one layer, eight vectors at a time: their pieces of
// 16 bytes are dealt out to its lanes one after another.  A kept vector's place is never
// behind its source (path rises), and eight are read before the first of them is written: no
// vector is overwritten before it was read.
//
// What bounds them, on MI355X: memory, behind three or four trips that a token's place takes (lengths, parents,
// page).  Append: 10766 tokens of 32 heads 24 us, 5.4 TB/s; 64 trees of up to 24 nodes, 128 heads 12.2 us, 3.4
// TB/s (with the vectors asked for before the angles 12.6); one token 3.4.  Keep: 61 layers of 64
// sequences of up to 24 nodes 10.9 us (13.2 where a wavefront took 64 pieces of every vector); one 4.1.
#include "common.hpp"

namespace sd {
namespace {

constexpr int kThreads = 256, kHeads = 4;

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  __device__ static float lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
  __device__ static float hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }
  __device__ static uint32_t pack(float lo, float hi) {
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    const x2 r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, r);
  }
};
struct F16 {
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  __device__ static float lo(uint32_t v) { return (float)__builtin_bit_cast(x2, v)[0]; }
  __device__ static float hi(uint32_t v) { return (float)__builtin_bit_cast(x2, v)[1]; }
  __device__ static uint32_t pack(float lo, float hi) {
    const x2 r = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, r);
  }
};

// Where token j of sequence b is cached, null for a place that does not exist.
__device__ __forceinline__ uint16_t* place_of(const Pages& p, int b, int64_t j) {
  if (j < 0 || j >= p.capacity) return nullptr;
  const int pg = p.table ? (int)j / p.page_size : 0;
  const int page = p.table ? p.table[(int64_t)b * p.table_stride + pg] : b;
  if (page < 0 || page >= p.n_pages) return nullptr;
  return p.cache + (int64_t)page * p.page_stride + ((int)j - pg * p.page_size) * p.token_stride;
}

// (cos a, sin a).
__device__ __forceinline__ float2 turn_of(double a) {
  constexpr double kTwoOverPi = 0x1.45f306dc9c883p-1, kHi = 0x1.921fb54442d18p+0, kLo = 0x1.1a62633145c07p-54;
  constexpr double magic = 0x1.8p52;  // a / (pi / 2) to the nearest whole number, its low bits the quadrant
  const double z = fma(a, kTwoOverPi, magic), k = z - magic;
  const float r = (float)fma(-k, kLo, fma(-k, kHi, a)), s = r * r;
  const uint32_t quadrant = (uint32_t)__builtin_bit_cast(uint64_t, z);
  float v = fmaf(s, 2.7557319e-6f, -1.9841270e-4f);
  v = fmaf(s, v, 8.3333333e-3f);
  v = fmaf(s, v, -1.6666667e-1f);
  v = fmaf(s * r, v, r);
  float c = fmaf(s, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(s, c, -1.3888889e-3f);
  c = fmaf(s, c, 4.1666667e-2f);
  c = fmaf(s, c, -0.5f);
  c = fmaf(s, c, 1.f);
  float2 t = quadrant & 1u ? make_float2(v, c) : make_float2(c, v);
  if ((quadrant + 1u) & 2u) t.x = -t.x;
  if (quadrant & 2u) t.y = -t.y;
  return t;
}

// Four pairs' elements, first and second elements of a pair in x and y, packed two by two.
struct Four {
  u32x2 x, y;
};
// Pairs 4 g .. 4 g + 3 of a rotary part.  PAIRS: eight elements in a row; HALVES: four and four.
__device__ __forceinline__ Four load_four(const uint16_t* p, int g, int half, bool halves) {
  if (halves) return Four{*reinterpret_cast<const u32x2*>(p + 4 * g), *reinterpret_cast<const u32x2*>(p + half + 4 * g)};
  const u32x4 v = *reinterpret_cast<const u32x4*>(p + 8 * g);
  return Four{u32x2{(v[0] & 0xffffu) | (v[1] << 16), (v[2] & 0xffffu) | (v[3] << 16)},
              u32x2{(v[0] >> 16) | (v[1] & 0xffff0000u), (v[2] >> 16) | (v[3] & 0xffff0000u)}};
}
__device__ __forceinline__ void store_four(uint16_t* p, int g, int half, bool halves, Four f) {
  if (halves) {
    *reinterpret_cast<u32x2*>(p + 4 * g) = f.x;
    *reinterpret_cast<u32x2*>(p + half + 4 * g) = f.y;
  } else {
    *reinterpret_cast<u32x4*>(p + 8 * g) =
        u32x4{(f.x[0] & 0xffffu) | (f.y[0] << 16), (f.x[0] >> 16) | (f.y[0] & 0xffff0000u),
              (f.x[1] & 0xffffu) | (f.y[1] << 16), (f.x[1] >> 16) | (f.y[1] & 0xffff0000u)};
  }
}
template <class T>
__device__ __forceinline__ Four turned(Four f, const float2 (&t)[4]) {
  Four o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float xl = T::lo(f.x[i]), xh = T::hi(f.x[i]), yl = T::lo(f.y[i]), yh = T::hi(f.y[i]);
    const float2 a = t[2 * i], b = t[2 * i + 1];
    o.x[i] = T::pack(xl * a.x - yl * a.y, xh * b.x - yh * b.y);
    o.y[i] = T::pack(xl * a.y + yl * a.x, xh * b.y + yh * b.x);
  }
  return o;
}

// Heads that one wavefront turns: its lanes are pairs' groups of four by heads.
__host__ __device__ inline int heads_a_part(int dr) { return dr ? 64 / (dr / 8) * kHeads : 1; }
__host__ __device__ inline int parts_of(int H, int dr) { return 1 + (dr ? (H + heads_a_part(dr) - 1) / heads_a_part(dr) : 0); }

template <class T>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int64_t tokens) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int parts = parts_of(a.H, a.dr);
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + w;
  const int64_t tok = unit / parts;
  const int part = (int)(unit - tok * parts);
  if (tok >= tokens) return;
  int b, i, n;
  if (a.cu) {
    // the last sequence that does not begin behind the token, in 64-way steps
    const int t = (int)tok;
    int lo = 0, left = a.B;
    while (left > 64) {
      const int step = (left + 63) / 64, at = lane * step;
      const uint64_t m = __ballot(at < left && a.cu[lo + (at < left ? at : 0)] <= t);
      const int k = m ? 63 - __clzll((long long)m) : 0;
      lo += k * step;
      left = min(step, left - k * step);
    }
    const uint64_t m = __ballot(lane < left && a.cu[lo + (lane < left ? lane : 0)] <= t);
    if (m == 0) return;
    b = lo + 63 - __clzll((long long)m);
    const int from = max(a.cu[b], 0), to = min(a.cu[b + 1], a.Q);
    if (t >= to) return;
    i = t - from;
    n = to - from;
  } else {
    b = (int)(tok / a.Q);
    i = (int)(tok - (int64_t)b * a.Q);
    n = a.rows ? min(max(a.rows[b], 0), a.Q) : a.Q;
    if (i >= n) return;
  }
  const int64_t first = (int64_t)max(a.lens[b], 0) - n;
  int depth = i;
  if (a.parents) {
    const int up = lane < a.Q ? a.parents[(int64_t)b * a.Q + lane] : -1;
    depth = 0;
    for (int j = i;; ++depth) {
      const int p = __builtin_amdgcn_readlane(up, j);
      if (p < 0 || p >= j) break;
      j = p;
    }
  }
  const int64_t seq = a.cu ? 0 : b, row = a.cu ? tok : i;
  const int groups = a.dr / 8, half = a.dr / 2;
  const int slots = groups ? 64 / groups : 1, slot = groups ? lane / groups : 0, g = groups ? lane - slot * groups : 0;
  float2 t[4];
  if (groups) {
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = turn_of((double)(first + depth) * a.freq[4 * g + k]);
  }
  if (part == 0) {
    uint16_t* to = place_of(a.pages, b, first + i);
    const uint16_t* from = a.latent + seq * a.ls.chain + row * a.ls.row;
    if (to && 8 * lane < a.dc) *reinterpret_cast<u32x4*>(to + 8 * lane) = *reinterpret_cast<const u32x4*>(from + 8 * lane);
    if (lane < groups) {
      const Four k = turned<T>(load_four(a.k_rope + seq * a.krs.chain + row * a.krs.row, g, half, a.halves), t);
      if (to) store_four(to + a.dc, g, half, a.halves, k);
      if (a.k_out) store_four(a.k_out + seq * a.kos.chain + row * a.kos.row, g, half, a.halves, k);
    }
    return;
  }
  if (slot >= slots) return;
  const uint16_t* q = a.q + seq * a.qs.seq + row * a.qs.row;
  uint16_t* out = a.q_out + seq * a.qos.seq + row * a.qos.row;
  const int h0 = (part - 1) * slots * kHeads + slot;
  Four f[kHeads];
#pragma unroll
  for (int k = 0; k < kHeads; ++k)
    if (h0 + k * slots < a.H) f[k] = load_four(q + (h0 + k * slots) * a.qs.head, g, half, a.halves);
#pragma unroll
  for (int k = 0; k < kHeads; ++k)
    if (h0 + k * slots < a.H) store_four(out + (h0 + k * slots) * a.qos.head, g, half, a.halves, turned<T>(f[k], t));
}

constexpr int kBatch = 8, kMost = 72;  // vectors that a wavefront holds at once; pieces of a vector

__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a, int64_t waves) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + w;
  if (unit >= waves) return;
  const int b = (int)(unit % a.B);
  const int64_t layer = unit / a.B;
  const int n = a.rows ? min(max(a.rows[b], 0), a.Q) : a.Q, tau = min(max(a.tau[b], 0), n);
  const int64_t first = (int64_t)max(a.lens[b], 0) - n;
  uint16_t* base = a.pages.cache;
  int before = -1, kept = 0;
  bool whole = true;
  // 64 rows at a time: a lane finds where one of them comes from and goes to
  for (int j0 = 0; j0 < tau && whole; j0 += 64) {
    const int j = j0 + lane, v = j < tau ? a.path[(int64_t)b * a.Q + j] : -1;
    int last = __shfl_up(v, 1);
    if (lane == 0) last = before;
    const uint64_t wrong = __ballot(j < tau && (v <= last || v >= n));
    const int count = min(wrong ? __ffsll((unsigned long long)wrong) - 1 : 64, tau - j0);
    whole = !wrong;
    before = __builtin_amdgcn_readlane(v, 63);
    kept += count;
    const uint16_t *from = nullptr, *to = nullptr;
    if (lane < count && v != j) {
      from = place_of(a.pages, b, first + v);
      to = place_of(a.pages, b, first + j);
    }
    const int64_t src = from && to ? from - base : -1, dst = from && to ? to - base : -1;
    uint16_t* mine = base + layer * a.layer_stride;
    for (int k0 = 0; k0 < count; k0 += kBatch) {
      u32x4 held[kBatch * kMost / 64];
      int64_t at[kBatch * kMost / 64];
#pragma unroll
      for (int i = 0; i < kBatch * kMost / 64; ++i) {
        const int id = 64 * i + lane, v = id / a.pieces, piece = id - v * a.pieces, k = k0 + v;
        const int64_t f = __shfl(src, k & 63), d = __shfl(dst, k & 63);
        at[i] = v < kBatch && k < count && f >= 0 ? d + 8 * piece : -1;
        if (at[i] >= 0) held[i] = *reinterpret_cast<const u32x4*>(mine + f + 8 * piece);
      }
#pragma unroll
      for (int i = 0; i < kBatch * kMost / 64; ++i)
        if (at[i] >= 0) *reinterpret_cast<u32x4*>(mine + at[i]) = held[i];
    }
  }
  if (a.new_lens && layer == 0 && lane == 0) a.new_lens[b] = (int)max(first + kept, (int64_t)0);
}

}  // namespace

int64_t append_groups(int64_t tokens, int H, int dr) {
  const int64_t waves = tokens * parts_of(H, dr);
  return (waves + kThreads / 64 - 1) / (kThreads / 64);
}
hipError_t append_launch(const AppendArgs& a, int64_t tokens, sd_type type, hipStream_t s) {
  const dim3 grid((unsigned)append_groups(tokens, a.H, a.dr));
  return type == SD_TYPE_BF16 ? launch_timed("latent_append", append_kernel<Bf16>, grid, dim3(kThreads), s, a, tokens)
                              : launch_timed("latent_append", append_kernel<F16>, grid, dim3(kThreads), s, a, tokens);
}

int64_t keep_groups(int layers, int B) { return ((int64_t)layers * B + kThreads / 64 - 1) / (kThreads / 64); }
hipError_t keep_launch(const KeepArgs& a, hipStream_t s) {
  const int64_t waves = (int64_t)a.layers * a.B;
  return launch_timed("latent_keep", keep_kernel, dim3((unsigned)keep_groups(a.layers, a.B)), dim3(kThreads),
                      s, a, waves);
}

}  // namespace sd
