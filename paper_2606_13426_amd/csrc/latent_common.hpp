// What the two forms of latent attention share: element types and their matrix
// instructions, LDS by byte offsets, loads that write LDS, and the order of a token's
// pieces there.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "bufio.hpp"
#include "common.hpp"
#include "wavered.hpp"

namespace sd {
namespace latent {

constexpr int kThreads = 256, kTile = 64;
constexpr float kLn2 = 0.69314718f;
constexpr int kRope = 64;  // columns of the rotary part, zero past d_rope

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  __device__ static f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  __device__ static f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  __device__ static uint32_t pack(float lo, float hi) {
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    const x2 r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, r);
  }
  __device__ static float value(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
  static constexpr uint32_t kExponent = 0x7f80, kOne = 0x3f80;  // all exponent bits set: an infinity or NaN
  static constexpr float kBelow = 0.f, kReach = 8.f;
};
struct F16 {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  __device__ static f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  __device__ static f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  __device__ static uint32_t pack(float lo, float hi) {
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    const x2 r = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, r);
  }
  __device__ static float value(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  static constexpr uint32_t kExponent = 0x7c00, kOne = 0x3c00;
  static constexpr float kBelow = 11.f, kReach = 15.f;
};

// A row's reference, in powers of 2: a weight is 2^{score - reference}.  It is set kBelow below the
// largest score so far and moves when one exceeds it by more than kReach, so that weights reach
// 2^kReach, harmless in float32 sums and in `type`.  fp16 has its normal range down to 2^-14 and steps of
// 2^-24 below: with the largest weight between 2^11 and 2^15 those down to 2^-25 of it
// keep half a step of 2^-11, and a smaller one loses 2^-36 of it at most (a reference at the largest score:
// 2^-14 and 2^-25, so that thousands of keys 17 nats below one of value 0 were a third
// off).  Scores of 2^20 and more, which are as coarse as an eighth, keep the margin of 2^8.
constexpr float kCoarse = 0x1p20f;
template <class T>
__device__ __forceinline__ float reference(float mx) {
  return T::kBelow > 0.f && fabsf(mx) < kCoarse ? mx - T::kBelow : mx;
}
template <class T>
__device__ __forceinline__ float reach(float m) {
  return m + (T::kReach > 8.f && fabsf(m) < kCoarse ? T::kReach : 8.f);
}

// Bits 15 and 31 of the result say which halves of v hold an infinity or NaN (one
// more at the lowest place of a full exponent carries into the cleared sign).
template <class T>
__device__ __forceinline__ uint32_t lawless(uint32_t v) {
  constexpr uint32_t kMask = T::kExponent * 0x10001u, kStep = (T::kExponent & -T::kExponent) * 0x10001u;
  return (v & kMask) + kStep;
}

// The permutation of a token's 16-byte pieces (on the low three bits of their
// number): eight tokens in a row have eight different ones, and so have the
// piece pairs of four tokens in a row.
__device__ __forceinline__ int perm(int token) { return ((token & 3) << 1) | ((token >> 2) & 1); }

// f(0), f(1), .. f(N - 1) with the numbers as types' values.
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, I + 1>(f);
  }
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// A load known to be from global memory.  (One that might be from LDS counts as both, and while
// it is pending every wait for an LDS read is a wait for all of them.)
template <class V, class P>
__device__ __forceinline__ V load_global(const P* p) {
  return *(const __attribute__((address_space(1))) V*)(uint64_t)p;
}

// Over lanes 16 and 32 apart (in every one of them the same bits).
__device__ __forceinline__ float across(float v, bool row32, bool max) {
  uint32_t a = __builtin_bit_cast(uint32_t, v), b = a;
  row32 ? swap32(a, b) : swap16(a, b);
  const float x = __builtin_bit_cast(float, a), y = __builtin_bit_cast(float, b);
  return max ? fmaxf(x, y) : x + y;
}
__device__ __forceinline__ float quarter_max(float v) { return across(across(v, false, true), true, true); }
__device__ __forceinline__ float quarter_sum(float v) { return across(across(v, false, false), true, false); }

// LDS by byte offsets: one base and immediate offsets for a lane's reads.
typedef __attribute__((address_space(3))) char* Lds;
__device__ __forceinline__ Lds lds_of(void* p) { return (Lds)p; }
template <class V>
__device__ __forceinline__ V lds_read(Lds p) {
  return *(__attribute__((address_space(3))) V*)p;
}
__device__ __forceinline__ u32x2 lds_read_tr(Lds p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}
// A barrier for what the wavefronts exchange through LDS themselves.  It does not wait
// for loads that write LDS, as __syncthreads does: those are in flight across it.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// 16 bytes a lane from global memory to LDS at dst + 16 lane (dst uniform).  In
// assembly, because the compiler takes a load that writes LDS for one that any LDS read
// behind it may have to wait for, and then waits for all reads in flight where it should
// for one.  Nothing is returned to registers; the caller waits for the loads (vmcnt)
// before a barrier.  The wait states are those of a scalar register written by a vector
// instruction, and of M0.
typedef const __attribute__((address_space(1))) char* Global;
__device__ __forceinline__ uint32_t lds_address(Lds p) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint64_t)p);
}
__device__ __forceinline__ void load_lds(Global src, Lds dst) {
  asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_address(dst)),
               "v"((uint64_t)src)
               : "memory", "m0");
}
// A view of global memory for loads that write LDS, in scalar registers.
__device__ __forceinline__ u32x4 lds_view(const void* base, int64_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), kBufferWord3};
}
// The same from byte `off` of a view to dst + STEP + 16 lane: one register an address,
// and none to compute.  on: all ones, or 0 for no load at all.
template <int STEP>
__device__ __forceinline__ void load_lds_view(u32x4 view, uint32_t off, uint32_t dst, uint64_t on) {
  asm volatile(
      "s_nop 1\n\ts_mov_b64 exec, %4\n\ts_add_i32 m0, %0, %1\n\ts_nop 0\n\t"
      "buffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b64 exec, -1" ::"s"(dst),
      "n"(STEP), "v"(off), "s"(view), "s"(on)
      : "memory", "m0", "scc");
}

}  // namespace latent
}  // namespace sd
