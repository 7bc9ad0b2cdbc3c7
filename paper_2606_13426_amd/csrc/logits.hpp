// Rows of logits over a vocabulary, read in slices that workgroups hold in
// registers (gfx950).
//
// A row of V elements starts anywhere its element type allows.  Its 16-byte
// vectors are counted from the last 16-byte address at or below its start, so
// every load but the two at the row's ends is a whole aligned vector; those two
// go element by element and read nothing outside the row.  Slice s of a row is
// the kThreads * E elements from vector s * kThreads * E / VEC on: vector k of a
// slice's thread t is number k * kThreads + t of the slice, so the elements of a
// thread rise with k, and a wavefront's loads are contiguous.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.hpp"

namespace sd {
namespace logits {

constexpr int kThreads = 256;
constexpr float kLowest = -3.402823466e38f;
constexpr double kLog2e = 1.44269504088896340736;

// Element types as the kernels see them: the bits, the bits of -inf, and the value
// as float32.
struct F32 {
  typedef float raw;
  static constexpr int kVec = 4;
  static constexpr raw kNone = -INFINITY;
  __device__ static float value(raw r) { return r; }
};
struct BF16 {
  typedef uint16_t raw;
  static constexpr int kVec = 8;
  static constexpr raw kNone = 0xff80;
  __device__ static float value(raw r) { return __builtin_bit_cast(float, (uint32_t)r << 16); }
};
struct F16 {
  typedef uint16_t raw;
  static constexpr int kVec = 8;
  static constexpr raw kNone = 0xfc00;
  __device__ static float value(raw r) { return (float)__builtin_bit_cast(_Float16, r); }
};

// Elements from the last 16-byte address at or below p to p.
template <class T>
__device__ __forceinline__ int lead(const typename T::raw* p) {
  return (int)(((uintptr_t)p & 15u) / sizeof(typename T::raw));
}

// The row position of element i of this thread's slice (negative, or V and
// above, outside the row).
template <class T, int E, int N = kThreads>
__device__ __forceinline__ int position(int slice, int a, int i) {
  return ((slice * (E / T::kVec) + i / T::kVec) * N + (int)threadIdx.x) * T::kVec + i % T::kVec - a;
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// The 16 bytes from byte 4 * words + 2 * half on of the 32 bytes (lo, hi).
__device__ __forceinline__ u32x4 funnel(u32x4 lo, u32x4 hi, int words, bool half) {
  uint32_t v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  if (words & 1)
#pragma unroll
    for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
  if (words & 2)
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = v[i + 2];
  if (half)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(v[i + 1], v[i], 2);
  return u32x4{v[0], v[1], v[2], v[3]};
}

// Vector k of this thread in slice `slice`, as position() counts it with the lead a, of
// the row p[0..V): its bits, -inf's outside the row.  A row whose own lead is another (the
// second of a pair) is read in its aligned vectors, two for each vector of positions, and
// shifted.
// STREAM: rows that no later kernel reads pass by the caches.
template <class T>
union Vec {
  u32x4 v;
  typename T::raw r[T::kVec];
};
template <class T, int E, bool STREAM = false, int N = kThreads>
__device__ __forceinline__ Vec<T> load_vector(const typename T::raw* __restrict__ p, int a, int V, int slice, int k) {
  constexpr int VEC = T::kVec;
  const int off = (lead<T>(p) - a) & (VEC - 1);  // elements from an aligned vector to a vector of positions
  const int e0 = position<T, E, N>(slice, a, k * VEC);
  Vec<T> w;
  if (off == 0 && e0 >= 0 && e0 + VEC <= V) {
    const u32x4* q = reinterpret_cast<const u32x4*>(p + e0);
    w.v = STREAM ? __builtin_nontemporal_load(q) : *q;
  } else if (off != 0 && e0 - off >= 0 && e0 - off + 2 * VEC <= V) {
    const u32x4* q = reinterpret_cast<const u32x4*>(p + (e0 - off));
    w.v = funnel(q[0], q[1], off * (int)sizeof(w.r[0]) >> 2, sizeof(w.r[0]) == 2 && (off & 1));
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      w.r[j] = T::kNone;
      if (e0 + j >= 0 && e0 + j < V) w.r[j] = p[e0 + j];
    }
  }
  return w;
}
// The slice's elements of this thread: x[i] is the one at position(i).
template <class T, int E, bool STREAM = false, int N = kThreads>
__device__ __forceinline__ void load_slice(const typename T::raw* __restrict__ p, int a, int V, int slice,
                                           float (&x)[E]) {
  constexpr int VEC = T::kVec, NV = E / VEC;
  Vec<T> w[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) w[k] = load_vector<T, E, STREAM, N>(p, a, V, slice, k);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[k * VEC + j] = T::value(w[k].r[j]);
}

// Slices of 256 * E elements that cover a row at any alignment.
inline int slices(int V, int E) { return (int)(((int64_t)V + 7 + (int64_t)kThreads * E - 1) / (kThreads * E)); }

// The elements a thread holds: 32, or 8 where rows of such slices would leave
// compute units without a workgroup (256 compute units, four workgroups each).
// In us, 8 / 32: one chain of 4 drafts over 32000 (bf16) 28 / 35, of 8 over 131072 35 / 47, 8
// of 8 67 / 69, 64 of 8 295 / 245, 32 of 5 over 50001 (f32) 51 / 61; log-probabilities of 16 rows of
// 131072 (bf16) 20 / 19, of 2048 306 / 161.
inline int per_thread(int64_t rows, int V) { return rows * slices(V, 32) >= 1024 ? 32 : 8; }

}  // namespace logits
}  // namespace sd
