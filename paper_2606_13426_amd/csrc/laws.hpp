// Laws over a vocabulary in float64: what the verifications of drafted tokens share.  A row's
// law is e^{(x - m) / T} / S; slices of a row (logits.hpp) are a workgroup's, which sums and
// searches them with the helpers below.
#pragma once

#include "common.hpp"
#include "logits.hpp"
#include "wavered.hpp"

namespace sd {
namespace laws {

using namespace logits;

// What a slice says of its part of a row.
struct Part {
  double S, U;  // sums against the slice's own maximum m: of the weights w, and of w (x - m), which log-probabilities need
  float m;      // -inf: nothing but -inf in it
  float pad;
};

__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp<kDppXor1>(v));
  v = fmaxf(v, dpp<kDppXor2>(v));
  v = fmaxf(v, dpp<kDppHalfMirror>(v));
  v = fmaxf(v, dpp<kDppMirror>(v));
  uint32_t a = __builtin_bit_cast(uint32_t, v), b = a;
  swap16(a, b);
  a = b = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  swap32(a, b);
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// The law's exponent: log2(e) / T, and the difference of logits below which a weight is 2^-1000 of the
// largest and less.
struct Scale {
  double c, low;
};
// 2^{d c} for d c in [-1001, 1] in float64, NaN for NaN: the whole part goes to the exponent (taken from the
// low bits of d c + 1.5 2^52, which end at the units), the rest, at most a half in size, to the
// Chebyshev expansion of 2^r on [-1/2, 1/2] up to its tenth term (3.2e-16 off), as a polynomial.
__device__ __forceinline__ double pow2(double d, double c) {
  constexpr double magic = 0x1.8p52;
  constexpr double k[11] = {1.0,
                            0x1.62e42fefa3a19p-1,
                            0x1.ebfbdff82c5aep-3,
                            0x1.c6b08d703ce43p-5,
                            0x1.3b2ab6fb9f1a3p-7,
                            0x1.5d87fe9d7afb3p-10,
                            0x1.430913112cb56p-13,
                            0x1.ffcb54047bef3p-17,
                            0x1.62bfc2c7ae40ep-20,
                            0x1.b675be272450dp-24,
                            0x1.e6228bff026d1p-28};
  const double z = fma(d, c, magic), r = fma(d, c, magic - z);
  double p = k[10];
#pragma unroll
  for (int i = 9; i >= 0; --i) p = fma(p, r, k[i]);
  return __builtin_amdgcn_ldexp(p, (int)(uint32_t)__builtin_bit_cast(uint64_t, z));
}
// e^{(x - m) / T} of one element, 0 below 2^-1000.
__device__ __forceinline__ double weight(float x, float m, Scale c) {
  const double d = (double)x - (double)m, v = pow2(d, c.c);
  return d < c.low ? 0.0 : v;
}
// The same with 2^-1000 for less and for NaN: for sums beside a weight of 1, whose caller looks for NaN.
__device__ __forceinline__ double weight_or_tiny(float x, float m, Scale c) {
  return pow2(fmax((double)x - (double)m, c.low), c.c);
}

// The maximum of a workgroup's slice x and the weights' sum against it (NaN where a value is NaN or +inf; U is 0, verification has no
// use for it), in float64 throughout: verification divides differences of two laws by one another.
template <class T, int E>
__device__ __forceinline__ Part slice_sums64(const float (&x)[E], Scale c, double* red, float* redm) {
  const int t = threadIdx.x, w = t >> 6;
  float m = x[0];
  bool nan = false;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    m = fmaxf(m, x[i]);
    nan |= x[i] != x[i];
  }
  m = wave_max(m);
  if ((t & 63) == 0) redm[w] = m;
  __syncthreads();
  m = fmaxf(fmaxf(redm[0], redm[1]), fmaxf(redm[2], redm[3]));
  double s[2] = {0.0, 0.0};
  if (m > -INFINITY) {
#pragma unroll
    for (int i = 0; i < E; ++i) s[i & 1] += weight_or_tiny(x[i], m, c);
  }
  const double v = wave_sum(nan || m == INFINITY ? NAN : s[0] + s[1]);
  if ((t & 63) == 0) red[w] = v;
  __syncthreads();
  return Part{red[0] + red[1] + (red[2] + red[3]), 0.0, m, 0.f};
}

// max(0, A wq - B wp), exactly 0 where the two are the same numbers (both products rounded).
__device__ __forceinline__ double excess_of(double A, double wq, double B, double wp) {
#pragma clang fp contract(off)
  const double q = A * wq, p = B * wp;
  return fmax(q - p, 0.0);
}

// Inclusive sums of v over the workgroup's threads, in their order.
__device__ __forceinline__ double block_scan(double v, double* red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  for (int i = 0; i < w; ++i) v += red[i];
  return v;
}
__device__ __forceinline__ double block_sum(double v, double* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return red[0] + red[1] + (red[2] + red[3]);
}
// The lowest thread whose flag is set, kThreads if none.
__device__ __forceinline__ int block_first(bool flag, int* red) {
  const uint64_t m = __ballot(flag);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
    red[threadIdx.x >> 6] = m ? (int)(threadIdx.x & ~63u) + __ffsll((unsigned long long)m) - 1 : kThreads;
  __syncthreads();
  return min(min(red[0], red[1]), min(red[2], red[3]));
}
__device__ __forceinline__ int block_last(bool flag, int* red) {
  const uint64_t m = __ballot(flag);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
    red[threadIdx.x >> 6] = m ? (int)(threadIdx.x & ~63u) + 63 - __clzll((long long)m) : -1;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}

// The workspace's parts, each at a multiple of 256 bytes.
inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

inline Scale scale_of(double inv_t) { return Scale{inv_t * kLog2e, -1000.0 / (inv_t * kLog2e)}; }

// f with the element type's tag.
template <class F>
auto by_type(sd_type type, F&& f) {
  return type == SD_TYPE_F32 ? f(F32{}) : type == SD_TYPE_BF16 ? f(BF16{}) : f(F16{});
}

}  // namespace laws
}  // namespace sd
