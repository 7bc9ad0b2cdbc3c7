// Laws over a vocabulary: log-probabilities of given tokens with entropy and
// alternatives, and the verification of drafted tokens (Alg. 6 / Alg. 2) with the
// draw of the next one.
//
// All of it streams rows of logits once or twice (logits.hpp): a workgroup holds
// a slice of a row in registers, so its maximum, sum, entropy term and largest
// elements come from one read, and a second kernel joins a row's slices.  With
// z = x / T and m the slice's maximum,
//   S = sum e^{(x - m) / T},   U = sum (x - m) e^{(x - m) / T}.
// Log-probabilities: differences and exponentials in float32 (one instruction each), the sums of a
// thread's elements too; everything across threads and slices is float64.  Verification is
// float64 from the difference on: with draft and target next to equal, h = v / (v + 1 - alpha) divides
// differences of the two laws, and an error of 1e-7 of them would be one of 1e-7 / (1 - alpha).
//
// What bounds it, on MI355X: verification's two passes over all rows by float64 products, 17
// instructions an element (64 chains of 8 drafts over 131072 bf16 tokens: sums 94 to 117 us from a
// cool to a warm card, 3.0 to 2.4 TB/s; excess 86 to 106 us; float32 exponentials ran at the stream's
// rate, 45 and 39), and so the draw's two passes over two rows a chain (18 to 22 and 33 to 39 us
// there); log-probabilities by vector instructions, about 14 an element with the alternatives (2048
// rows of 131072 bf16: 145 us, 3.7 TB/s, 119 of them issuing).  Few rows are launches and trips to
// memory: one row of 32000 takes 8 us in one kernel, one chain of 4 drafts 24 us in five.
#include "common.hpp"
#include "laws.hpp"
#include "logits.hpp"
#include "philox.hpp"
#include "wavered.hpp"

namespace sd {
namespace {

using namespace laws;
using laws::wave_max;  // beside the one of keys below

// ------------------------------------------------------------ alternatives --
// Elements are ordered by keys: the value's bits in an order-preserving form
// above, the complement of the position below, so equal values fall by position
// and no two elements share a key.  0 stands for no element.
__device__ __forceinline__ uint64_t key_of(float x, int pos) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // -0 and 0 are equal
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return ((uint64_t)o << 32) | (uint32_t)~pos;
}
__device__ __forceinline__ int key_pos(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, o ^ ((uint32_t)((int32_t)~o >> 31) | 0x80000000u));
}
template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {
  return ((uint64_t)dpp32<CTRL>((uint32_t)(v >> 32)) << 32) | dpp32<CTRL>((uint32_t)v);
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t lane_key(uint64_t v, int i) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, i);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  v = max64(v, dpp64<kDppXor1>(v));
  v = max64(v, dpp64<kDppXor2>(v));
  v = max64(v, dpp64<kDppHalfMirror>(v));
  v = max64(v, dpp64<kDppMirror>(v));
  v = max64(v, (uint64_t)__shfl_xor((unsigned long long)v, 16));
  return max64(v, (uint64_t)__shfl_xor((unsigned long long)v, 32));
}

constexpr int kPool = 1024;  // candidates a workgroup orders at once
struct TopLds {
  uint64_t group[64];
  float groupf[64];
  uint64_t pool[kPool];
  uint64_t bound;
  float boundf;
  int count;
};

// The keys of pool[0..c) in falling order to out[0..n) (fewer than n: the rest 0).
// Every key counts those above it; c is mostly little more than n.
template <int N = kThreads>
__device__ __forceinline__ void write_ranked(const uint64_t* pool, int c, int n, uint64_t* out) {
  for (int i = threadIdx.x; i < c; i += N) {
    const uint64_t k = pool[i];
    int above = 0;
    for (int j = 0; j < c; ++j) above += pool[j] > k;
    if (above < n) out[above] = k;
  }
  for (int i = c + (int)threadIdx.x; i < n; i += N) out[i] = 0;
}

// The n largest of the slice x to out[0..n) in falling order, 0 past its elements; best[k] is
// the largest of vector k of this thread.  The largest values of 64 groups of threads give a
// bound: n groups hold one at or above the n-th largest of them, so the n largest elements
// are among those not below it, which are few: most wavefronts find no candidate in a
// compare or two an element.  Where equal values overflow the pool (few values that are
// not -inf, a constant row) the groups' largest keys give the bound, which no two
// elements share, and where that overflows it too (an order made for it) the n largest
// are taken one after another.
template <class T, int E, int N = kThreads>
__device__ __forceinline__ void slice_top(const float (&x)[E], const float (&best)[E / T::kVec], int slice, int a, int V, int n, TopLds& sm,
                                          uint64_t* out) {
  constexpr int G = N / 64;  // threads a group
  static_assert(G == 4 || G == 16, "groups of lanes side by side");
  const int t = threadIdx.x;
  float g = best[0];
#pragma unroll
  for (int k = 1; k < E / T::kVec; ++k) g = fmaxf(g, best[k]);
  g = fmaxf(g, dpp<kDppXor1>(g));
  g = fmaxf(g, dpp<kDppXor2>(g));
  if (G == 16) {
    g = fmaxf(g, dpp<kDppHalfMirror>(g));
    g = fmaxf(g, dpp<kDppMirror>(g));
  }
  if (t % G == 0) sm.groupf[t / G] = g;
  if (t == 0) sm.count = 0;
  __syncthreads();
  if (t < 64) {
    const float k = sm.groupf[t];
    int from = 0;  // groups not below this one
#pragma unroll
    for (int i = 0; i < 64; ++i)
      from += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, k), i)) >= k;
    const float b = wave_max(from >= n ? k : -INFINITY);
    if (t == 0) sm.boundf = b;
  }
  __syncthreads();
  const float boundf = sm.boundf;
  if (boundf > -INFINITY) {
#pragma unroll
    for (int k = 0; k < E / T::kVec; ++k)
      if (__any(best[k] >= boundf))
#pragma unroll
        for (int i = k * T::kVec; i < (k + 1) * T::kVec; ++i) {
          if (!__any(x[i] >= boundf)) continue;
          const int pos = position<T, E, N>(slice, a, i);
          if (x[i] >= boundf && pos >= 0 && pos < V) {
            const int c = atomicAdd(&sm.count, 1);
            if (c < kPool) sm.pool[c] = key_of(x[i], pos);
          }
        }
    __syncthreads();
    const int c = sm.count;
    if (c <= kPool) {
      write_ranked<N>(sm.pool, c, n, out);
      return;
    }
  }
  uint64_t mine = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int pos = position<T, E, N>(slice, a, i);
    if (pos >= 0 && pos < V) mine = max64(mine, key_of(x[i], pos));
  }
  uint64_t gk = max64(mine, dpp64<kDppXor1>(mine));
  gk = max64(gk, dpp64<kDppXor2>(gk));
  if (G == 16) {
    gk = max64(gk, dpp64<kDppHalfMirror>(gk));
    gk = max64(gk, dpp64<kDppMirror>(gk));
  }
  __syncthreads();
  if (t % G == 0) sm.group[t / G] = gk;
  if (t == 0) sm.count = 0;
  __syncthreads();
  if (t < 64) {
    const uint64_t k = sm.group[t];
    int above = 0;
    for (int i = 0; i < 64; ++i) above += lane_key(k, i) > k;
    // groups without an element share the key 0: their rank is the first of them
    const uint64_t at = __ballot(above == n - 1);
    const uint64_t b = at ? lane_key(k, __ffsll((unsigned long long)at) - 1) : 0;
    if (t == 0) sm.bound = b;
  }
  __syncthreads();
  const uint64_t bound = sm.bound;
  if (mine != 0 && mine >= bound) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int pos = position<T, E, N>(slice, a, i);
      if (pos < 0 || pos >= V) continue;
      const uint64_t k = key_of(x[i], pos);
      if (k < bound) continue;
      const int c = atomicAdd(&sm.count, 1);
      if (c < kPool) sm.pool[c] = k;
    }
  }
  __syncthreads();
  const int c = sm.count;
  if (c <= kPool) {
    write_ranked<N>(sm.pool, c, n, out);
    return;
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < n; ++r) {
    uint64_t k = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int pos = position<T, E, N>(slice, a, i);
      const uint64_t q = pos >= 0 && pos < V ? key_of(x[i], pos) : 0;
      if (q < last) k = max64(k, q);
    }
    k = wave_max(k);
    __syncthreads();
    if ((t & 63) == 0) sm.group[t >> 6] = k;
    __syncthreads();
    k = sm.group[0];
    for (int i = 1; i < N / 64; ++i) k = max64(k, sm.group[i]);
    if (t == 0) out[r] = k;
    last = k;
  }
}

// ------------------------------------------------------------------- sums --
// Sums of a workgroup's slice: m its maximum, S and U; best[k] the largest of vector k of this thread.
template <int W>
__device__ __forceinline__ double pairwise(const double* p) {
  if constexpr (W == 1) return p[0];
  else return pairwise<W / 2>(p) + pairwise<W / 2>(p + W / 2);
}
template <class T, int E, int N = kThreads>
__device__ __forceinline__ Part slice_sums(const float (&x)[E], float c, double* red, float* redm,
                                           float (&best)[E / T::kVec]) {
  const int t = threadIdx.x, w = t >> 6;
  constexpr int NV = E / T::kVec, W = N / 64;
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    best[k] = x[k * T::kVec];
#pragma unroll
    for (int j = 1; j < T::kVec; ++j) best[k] = fmaxf(best[k], x[k * T::kVec + j]);
    m = fmaxf(m, best[k]);
  }
  m = wave_max(m);
  if ((t & 63) == 0) redm[w] = m;
  __syncthreads();
  m = redm[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, redm[i]);
  const float ref = m == -INFINITY ? 0.f : m;
  float s[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = x[i] - ref;
    const float e = __builtin_amdgcn_exp2f(d * c);
    s[i & 3] += e;
    u[i & 3] = __fmaf_rn(e, fmaxf(d, kLowest), u[i & 3]);
  }
  const double S = (double)s[0] + s[1] + ((double)s[2] + s[3]), U = (double)u[0] + u[1] + ((double)u[2] + u[3]);
  // the lower lanes add up the one, the upper lanes the other
  const double v = group_sum(swap_add<true>(S, U), 32);
  if ((t & 31) == 0) red[(t & 32 ? W : 0) + w] = v;
  __syncthreads();
  Part p;
  p.S = pairwise<W>(red);
  p.U = pairwise<W>(red + W);
  p.m = m;
  p.pad = 0.f;
  return p;
}

template <class T, int E>
__global__ __launch_bounds__(kThreads, 4) void logprobs_slice_kernel(const typename T::raw* __restrict__ x, int64_t ld,
                                                                  int V, int S, float c, int n,
                                                                  Part* __restrict__ parts,
                                                                  uint64_t* __restrict__ keys) {
  __shared__ double red[8];
  __shared__ float redm[4];
  __shared__ TopLds top;
  const int64_t id = blockIdx.x;
  const int slice = (int)(id % S);
  const typename T::raw* p = x + (id / S) * ld;
  const int a = lead<T>(p);
  float v[E], best[E / T::kVec];
  load_slice<T, E, true>(p, a, V, slice, v);
  const Part r = slice_sums<T, E>(v, c, red, redm, best);
  if (threadIdx.x == 0) parts[id] = r;
  if (n > 0) slice_top<T, E>(v, best, slice, a, V, n, top, keys + id * n);
}

// What a row's sums say, by a workgroup of N threads: the given tokens, and the alternatives whose keys are in
// best[0..n) (LDS, behind a barrier).
template <class T, int N = kThreads>
__device__ __forceinline__ void write_row(const typename T::raw* __restrict__ x, int64_t ld, int V, double inv_t,
                                          int64_t row, float m, double s, double u, int n_tok,
                                          const int32_t* __restrict__ tokens, float* __restrict__ logprob,
                                          float* __restrict__ entropy, float* __restrict__ lse, int n,
                                          int32_t* __restrict__ ids, float* __restrict__ tops, const uint64_t* best) {
  const int t = threadIdx.x;
  const bool law = s > 0.0 && isfinite(s), none = s == 0.0;
  const double logs = log(s);
  auto logp = [&](float v) {
    return law ? (float)(((double)v - (double)m) * inv_t - logs) : none ? -INFINITY : NAN;
  };
  if (t == 0) {
    if (lse) lse[row] = law ? (float)((double)m * inv_t + logs) : none ? -INFINITY : NAN;
    if (entropy) entropy[row] = law ? (float)(logs - u * inv_t / s) : none ? 0.f : NAN;
  }
  for (int i = t; i < n_tok; i += N) {
    const int tok = tokens[row * n_tok + i];
    logprob[row * n_tok + i] = logp(tok >= 0 && tok < V ? T::value(x[row * ld + tok]) : -INFINITY);
  }
  if (t < n) {
    const uint64_t me = best[t];
    const bool real = me != 0 && (law || none);
    ids[row * n + t] = real ? key_pos(me) : -1;
    tops[row * n + t] = law || none ? (me != 0 ? logp(key_value(me)) : -INFINITY) : NAN;
  }
}

// A row that one workgroup holds at once: all of it in one kernel.
constexpr int kRowThreads = 1024;
template <class T, int E>
__global__ __launch_bounds__(kRowThreads) void logprobs_row_kernel(
    const typename T::raw* __restrict__ x, int64_t ld, int V, float c, double inv_t, int n_tok,
    const int32_t* __restrict__ tokens, float* __restrict__ logprob, float* __restrict__ entropy,
    float* __restrict__ lse, int n, int32_t* __restrict__ ids, float* __restrict__ tops) {
  __shared__ double red[2 * kRowThreads / 64];
  __shared__ float redm[kRowThreads / 64];
  __shared__ TopLds top;
  __shared__ uint64_t keys[SD_MAX_TOP];
  const int64_t row = blockIdx.x;
  const typename T::raw* p = x + row * ld;
  const int a = lead<T>(p);
  float v[E], best[E / T::kVec];
  load_slice<T, E, true, kRowThreads>(p, a, V, 0, v);
  const Part r = slice_sums<T, E, kRowThreads>(v, c, red, redm, best);
  if (n > 0) {
    slice_top<T, E, kRowThreads>(v, best, 0, a, V, n, top, keys);
    __syncthreads();
  }
  write_row<T, kRowThreads>(x, ld, V, inv_t, row, r.m, r.S, r.U, n_tok, tokens, logprob, entropy, lse, n, ids, tops,
                            keys);
}

// One workgroup a row: the slices' sums, the given tokens and the alternatives.
template <class T>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(
    const typename T::raw* __restrict__ x, int64_t ld, int V, int S, double inv_t, int n_tok,
    const int32_t* __restrict__ tokens, float* __restrict__ logprob, float* __restrict__ entropy,
    float* __restrict__ lse, int n, int32_t* __restrict__ ids, float* __restrict__ tops,
    const Part* __restrict__ parts, const uint64_t* __restrict__ keys) {
  __shared__ double red[8];
  __shared__ float redm[4];
  __shared__ TopLds top;
  __shared__ uint64_t best[SD_MAX_TOP];
  const int t = threadIdx.x, w = t >> 6;
  const int64_t row = blockIdx.x;
  const Part* p = parts + row * S;
  float m = -INFINITY;
  for (int i = t; i < S; i += kThreads) m = fmaxf(m, p[i].m);
  m = wave_max(m);
  if ((t & 63) == 0) redm[w] = m;
  __syncthreads();
  m = fmaxf(fmaxf(redm[0], redm[1]), fmaxf(redm[2], redm[3]));
  double s = 0.0, u = 0.0;
  for (int i = t; i < S; i += kThreads) {
    const Part q = p[i];
    if (q.m == -INFINITY && q.S == 0.0) continue;  // nothing in it (a NaN leaves S NaN)
    const double d = (double)q.m - (double)m, f = exp(d * inv_t);
    s += q.S * f;
    u += f == 0.0 ? 0.0 : f * (q.U + d * q.S);
  }
  s = wave_sum(s);
  u = wave_sum(u);
  if ((t & 63) == 0) {
    red[w] = s;
    red[4 + w] = u;
  }
  __syncthreads();
  s = red[0] + red[1] + (red[2] + red[3]);
  u = red[4] + red[5] + (red[6] + red[7]);
  auto finish = [&]() {
    write_row<T>(x, ld, V, inv_t, row, m, s, u, n_tok, tokens, logprob, entropy, lse, n, ids, tops, best);
  };
  if (n == 0) {
    finish();
    return;
  }
  // The slices' lists are ordered: the n-th largest of their first q elements, q
  // the least with S q >= n, bounds the n largest of all from below.
  const uint64_t* k = keys + row * S * n;
  const int q = (n + S - 1) / S, pool = min(S * q, kPool);
  for (int i = t; i < pool; i += kThreads) top.pool[i] = k[(int64_t)(i / q) * n + i % q];
  if (t == 0) {
    top.count = 0;
    top.bound = 0;
  }
  __syncthreads();
  for (int i = t; i < pool; i += kThreads) {
    const uint64_t me = top.pool[i];
    int above = 0;
    for (int j = 0; j < pool; ++j) above += top.pool[j] > me;
    if (above == n - 1) top.bound = me;
  }
  __syncthreads();
  const uint64_t bound = top.bound > 0 ? top.bound : 1;
  __syncthreads();
  for (int i = t; i < S; i += kThreads)
    for (int j = 0; j < n; ++j) {
      const uint64_t me = k[(int64_t)i * n + j];
      if (me < bound) break;
      const int c = atomicAdd(&top.count, 1);
      if (c < kPool) top.pool[c] = me;
    }
  __syncthreads();
  if (top.count <= kPool) {
    write_ranked(top.pool, top.count, n, best);
  } else {
    // more than kPool lists, whose heads gave a weak bound: one after another
    uint64_t last = ~0ull;
    for (int r = 0; r < n; ++r) {
      uint64_t me = 0;
      for (int64_t i = t; i < (int64_t)S * n; i += kThreads)
        if (k[i] < last) me = max64(me, k[i]);
      me = wave_max(me);
      __syncthreads();
      if ((t & 63) == 0) top.group[w] = me;
      __syncthreads();
      last = max64(max64(top.group[0], top.group[1]), max64(top.group[2], top.group[3]));
      if (t == 0) best[r] = last;
    }
  }
  __syncthreads();
  finish();
}

// ------------------------------------------------------------ verification --
// Rows of a chain in the order the workspace holds them: target rows 0..K, then
// draft rows 0..K-1.
struct Rows {
  const void *draft, *target;
  sd_stride ds, ts;
};
template <class T>
__device__ __forceinline__ const typename T::raw* row_of(const Rows& r, int b, int i, int K) {
  return i <= K ? reinterpret_cast<const typename T::raw*>(r.target) + (int64_t)b * r.ts.chain + (int64_t)i * r.ts.row
                : reinterpret_cast<const typename T::raw*>(r.draft) + (int64_t)b * r.ds.chain +
                      (int64_t)(i - K - 1) * r.ds.row;
}
__device__ __forceinline__ int drafts(const int32_t* kb, int b, int K) { return min(max(kb[b], 0), K); }

// A row's law: e^{(x - m) c} / S with c = log2(e) / T, log S in float64.  S is 0 where the row is all
// -inf and NaN where it has no law.
struct Law {
  double S, logS;
  float m, pad;
};
struct Mass {
  double q, p;
};

// Sums of every valid row's slices.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(Rows rows, int K, int V, int S, Scale c,
                                                               const int32_t* __restrict__ kb,
                                                               Part* __restrict__ parts) {
  __shared__ double red[4];
  __shared__ float redm[4];
  const int64_t id = blockIdx.x;
  const int slice = (int)(id % S), r = (int)(id / S), b = r / (2 * K + 1), i = r % (2 * K + 1);
  const int n = drafts(kb, b, K);
  if (n == 0 || (i <= K ? i > n : i - K - 1 >= n)) return;
  const typename T::raw* p = row_of<T>(rows, b, i, K);
  float v[E];
  load_slice<T, E>(p, lead<T>(p), V, slice, v);
  const Part q = slice_sums64<T, E>(v, c, red, redm);
  if (threadIdx.x == 0) parts[id] = q;
}

// Token verification's tau from the coins of n drafts.
__device__ __forceinline__ int first_rejected(uint64_t cm, int n) {
  const uint64_t rej = ~cm & (n >= 64 ? ~0ull : (1ull << n) - 1ull);
  return rej ? __ffsll((unsigned long long)rej) : n + 1;
}

// One workgroup a chain: the rows' laws (16 lanes a row), the log-ratios, log alpha_j; with
// token verification also the decision.
template <class T>
__global__ __launch_bounds__(kThreads) void verify_join_kernel(Rows rows, int K, int V, int S, int mode, double inv_t,
                                                         const int32_t* __restrict__ tokens,
                                                         const int32_t* __restrict__ kb,
                                                         const double* __restrict__ uniforms,
                                                         const uint32_t* __restrict__ round, uint64_t seed,
                                                         const Part* __restrict__ parts, Law* __restrict__ laws,
                                                         double* __restrict__ la, int32_t* __restrict__ tau,
                                                         float* __restrict__ lar, float* __restrict__ ratio,
                                                         uint64_t* __restrict__ coins) {
  __shared__ Law law[2 * SD_MAX_BLOCK + 1];
  const int b = blockIdx.x, t = threadIdx.x, lane = t, in = t & 15;
  const int n = drafts(kb, b, K);
  // the draft's two logits are on their way while the rows' sums are joined
  const int tok = lane < n ? tokens[(int64_t)b * K + lane] : -1;
  const bool known = tok >= 0 && tok < V;
  float xq = -INFINITY, xp = -INFINITY;
  if (known) {
    xq = T::value(row_of<T>(rows, b, lane, K)[tok]);
    xp = T::value(row_of<T>(rows, b, K + 1 + lane, K)[tok]);
  }
  if (n > 0)
    for (int i = t >> 4; i < 2 * K + 1; i += kThreads / 16) {
      if (i <= K ? i > n : i - K - 1 >= n) continue;
      const Part* p = parts + ((int64_t)b * (2 * K + 1) + i) * S;
      float m = -INFINITY;
      for (int s = in; s < S; s += 16) m = fmaxf(m, p[s].m);
      m = (float)group_max((double)m, 16);
      double sum = 0.0;
      for (int s = in; s < S; s += 16) {
        const Part q = p[s];
        if (!(q.m == -INFINITY && q.S == 0.0)) sum += q.S * exp(((double)q.m - (double)m) * inv_t);
      }
      sum = group_sum(sum, 16);
      if (in == 0) {
        law[i] = Law{sum, log(sum), m, 0.f};
        laws[(int64_t)b * (2 * K + 1) + i] = law[i];
      }
    }
  __syncthreads();
  if (t >= 64) return;
  // The log-ratio of draft j = lane + 1: -inf where q has nothing for the draft, whatever p has.  Rows of
  // the same values (up to one offset) give exactly the same (x - m) / T; their sums differ by the
  // order in which they were added, since rows start at other places of a 16-byte vector: at most
  // 160 roundings each (the largest vocabulary's 2049 slices by 16 lanes, 25 inside a slice), 2^-44.6 of
  // their ratio.  So less than kSame is a ratio of 1, and an alpha that near to 1 is 1: its h_j is then 1
  // and not a quotient of roundings.
  constexpr double kSame = 0x1p-44;
  double ell = NAN;
  if (lane < n) {
    const Law &lq = law[lane], &lp = law[K + 1 + lane];
    const bool okq = lq.S >= 0.0 && isfinite(lq.S), okp = lp.S >= 0.0 && isfinite(lp.S);
    if (okq && okp) {
      if (lq.S == 0.0 || xq == -INFINITY)
        ell = -(double)INFINITY;
      else if (lp.S == 0.0 || xp == -INFINITY)
        ell = (double)INFINITY;
      else
        ell = (((double)xq - (double)lq.m) * inv_t - ((double)xp - (double)lp.m) * inv_t) - (lq.logS - lp.logS);
      if (fabs(ell) < kSame) ell = 0.0;
    }
  }
  const double use = ell == ell ? ell : -(double)INFINITY;  // no law: rejected
  double acc = 0.0, mine = 0.0;
  for (int i = 0; i < n; ++i) {
    const double e = __shfl(use, i);
    acc = acc == -(double)INFINITY ? acc : fmin(0.0, acc + e);
    if (acc > -kSame) acc = 0.0;
    if (i == lane) mine = acc;
  }
  if (lane < K) {
    ratio[(int64_t)b * K + lane] = lane < n ? (float)ell : 0.f;
    la[(int64_t)b * K + lane] = mine;
  }
  if (mode == SD_TOKEN || n == 0) {
    double eta = 2.0;
    if (lane < n) {
      if (uniforms) {
        eta = uniforms[(int64_t)b * (K + 1) + lane];
      } else {
        const uint4 w = philox((uint32_t)(lane >> 2), (uint32_t)b, round[b], TAG_COIN << 24, seed);
        eta = uniform64(pick(w, lane & 3));
      }
    }
    const uint64_t cm = __ballot(lane < n && eta < exp(fmin(0.0, use)));
    if (lane == 0) {
      tau[b] = n == 0 ? 0 : first_rejected(cm, n);
      lar[b] = 0.f;
      if (coins) coins[b] = n == 0 ? 0 : cm;
    }
  }
}

// The slices of v_j for j = 1..K_b - 1: rows j (0-based) of target and draft.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void verify_excess_kernel(Rows rows, int K, int V, int S, Scale c,
                                                                 const int32_t* __restrict__ kb,
                                                                 const Law* __restrict__ laws,
                                                                 const double* __restrict__ la,
                                                                 double* __restrict__ excess) {
  __shared__ double red[4];
  const int64_t id = blockIdx.x;
  const int slice = (int)(id % S), r = (int)(id / S), b = r / (K - 1), j = r % (K - 1) + 1;
  if (j >= drafts(kb, b, K)) return;
  const Law q = laws[(int64_t)b * (2 * K + 1) + j], p = laws[(int64_t)b * (2 * K + 1) + K + 1 + j];
  const double A = q.S == 0.0 ? 0.0 : exp(la[(int64_t)b * K + j - 1]) / q.S;
  const double B = p.S == 0.0 ? 0.0 : 1.0 / p.S;
  const float mq = q.S == 0.0 ? 0.f : q.m, mp = p.S == 0.0 ? 0.f : p.m;
  const typename T::raw *pq = row_of<T>(rows, b, j, K), *pp = row_of<T>(rows, b, K + 1 + j, K);
  float x[E], y[E];
  const int a = lead<T>(pq);
  load_slice<T, E>(pq, a, V, slice, x);
  load_slice<T, E>(pp, a, V, slice, y);
  double s[2] = {0.0, 0.0};
#pragma unroll
  for (int i = 0; i < E; ++i) s[i & 1] += excess_of(A, weight_or_tiny(x[i], mq, c), B, weight_or_tiny(y[i], mp, c));
  const double sum = wave_sum(isfinite(A) && isfinite(B) ? s[0] + s[1] : NAN);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) excess[((int64_t)b * K + j) * S + slice] = red[0] + red[1] + (red[2] + red[3]);
}

// Block verification's coins and tau of a chain with n > 0 drafts, by the whole workgroup: 16
// lanes add up the slices of a v_j.  The same bits in every workgroup that asks; `write`
// says which one puts them out.
__device__ __forceinline__ int decide(int b, int n, int K, int S, const double* __restrict__ uniforms,
                                      const uint32_t* __restrict__ round, uint64_t seed, const double* __restrict__ la,
                                      const double* __restrict__ excess, bool write, int32_t* __restrict__ tau,
                                      float* __restrict__ lar, uint64_t* __restrict__ coins) {
  __shared__ double vs[SD_MAX_BLOCK];
  __shared__ int tau_s;
  const int t = threadIdx.x, lane = t, in = t & 15;
  for (int j = 1 + (t >> 4); j < n; j += kThreads / 16) {
    const double* e = excess + ((int64_t)b * K + j) * S;
    double v = 0.0;
    for (int s = in; s < S; s += 16) v += e[s];
    v = group_sum(v, 16);
    if (in == 0) vs[j] = v;
  }
  __syncthreads();
  if (t < 64) {
    double l = 0.0, h = 0.0, eta = 2.0;
    if (lane < n) {
      l = la[(int64_t)b * K + lane];
      h = lane + 1 == n ? exp(l) : l >= 0.0 ? 1.0 : vs[lane + 1] / (vs[lane + 1] - expm1(l));
      if (uniforms) {
        eta = uniforms[(int64_t)b * (K + 1) + lane];
      } else {
        const uint4 w = philox((uint32_t)(lane >> 2), (uint32_t)b, round[b], TAG_COIN << 24, seed);
        eta = uniform64(pick(w, lane & 3));
      }
    }
    const uint64_t cm = __ballot(lane < n && eta < h);
    const int at = cm ? 65 - __clzll((long long)cm) : 1;
    const double res = at >= 2 ? __shfl(l, at - 2) : 0.0;
    if (lane == 0) {
      tau_s = at;
      if (write) {
        tau[b] = at;
        lar[b] = (float)res;
        if (coins) coins[b] = cm;
      }
    }
  }
  __syncthreads();
  return tau_s;
}

// ---------------------------------------------------------------- the draw --
// All of it in float64: a cumulative sum over a vocabulary is compared with a
// uniform, and the tokens' borders are as near as 1e-6 of the whole.
template <class T>
struct Pair {
  const typename T::raw *q, *p;  // the target's row tau - 1, the draft's (null where every draft was accepted)
  int iq, ip;                    // their places among the chain's rows
  bool any;
};
template <class T>
__device__ __forceinline__ Pair<T> drawn_rows(const Rows& rows, int b, int K, int n, int tau) {
  Pair<T> r{nullptr, nullptr, tau - 1, K + tau, n > 0};
  if (!r.any) return r;
  r.q = row_of<T>(rows, b, tau - 1, K);
  if (tau <= n) r.p = row_of<T>(rows, b, K + tau, K);
  return r;
}

// Slices of the two rows' sums, behind block verification's decision where there is one (excess).
template <class T, int E>
__global__ __launch_bounds__(kThreads) void draw_sums_kernel(
    Rows rows, int K, int V, int S, Scale c, const int32_t* __restrict__ kb, const double* __restrict__ uniforms,
    const uint32_t* __restrict__ round, uint64_t seed, const Law* __restrict__ laws, const double* __restrict__ la,
    const double* __restrict__ excess, int Se, int32_t* __restrict__ tau, float* __restrict__ lar,
    uint64_t* __restrict__ coins, Mass* __restrict__ sums, uint32_t* __restrict__ arrived) {
  __shared__ double red[8];
  const int slice = blockIdx.x % S, b = blockIdx.x / S, t = threadIdx.x;
  const int n = drafts(kb, b, K);
  if (slice == 0 && t == 0) arrived[b] = 0;
  if (n == 0) return;
  const int at = excess ? decide(b, n, K, Se, uniforms, round, seed, la, excess, slice == 0, tau, lar, coins) : tau[b];
  const Pair<T> r = drawn_rows<T>(rows, b, K, n, at);
  const int a = lead<T>(r.q);
  double s[2] = {0.0, 0.0};
  // (loops that are not unrolled: 20 KB of float64 code that every workgroup runs through once
  // would wait for its instructions)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const typename T::raw* p = h ? r.p : r.q;
    if (!p) continue;
    const Law& law = laws[(int64_t)b * (2 * K + 1) + (h ? r.ip : r.iq)];
    if (law.S == 0.0) continue;  // (a row of -inf alone; with a NaN among them S is NaN, and so is its sum here)
    const float m = law.m;
    Vec<T> x = load_vector<T, E>(p, a, V, slice, 0);
#pragma unroll 1
    for (int k = 0; k < E / T::kVec; ++k) {
      const Vec<T> next = k + 1 < E / T::kVec ? load_vector<T, E>(p, a, V, slice, k + 1) : x;
#pragma unroll
      for (int j = 0; j < T::kVec; ++j) s[h] += weight(T::value(x.r[j]), m, c);
      x = next;
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    s[h] = wave_sum(s[h]);
    if ((t & 63) == 0) red[4 * h + (t >> 6)] = s[h];
  }
  __syncthreads();
  if (t == 0)
    sums[blockIdx.x] = Mass{red[0] + red[1] + (red[2] + red[3]), red[4] + red[5] + (red[6] + red[7])};
}

// The factors of the residual law's two terms: w = max(0, A e^{(x - mq) / T} - B e^{(y - mp) / T}).
struct Residual {
  double A, B;
  float mq, mp;
};
// Every thread of the workgroup takes part and gets the same bits.
template <class T>
__device__ __forceinline__ Residual residual_of(const Pair<T>& r, int b, int K, int S, int mode, int tau,
                                                const Law* __restrict__ laws, const double* __restrict__ la,
                                                const Mass* __restrict__ sums, double* red) {
  double q = 0.0, p = 0.0;
  for (int i = threadIdx.x; i < S; i += kThreads) {
    q += sums[(int64_t)b * S + i].q;
    p += sums[(int64_t)b * S + i].p;
  }
  q = block_sum(q, red);
  p = block_sum(p, red);
  const double res = mode == SD_BLOCK && tau >= 2 ? la[(int64_t)b * K + tau - 2] : 0.0;
  Residual f;
  f.A = q == 0.0 ? 0.0 : exp(res) / q;
  f.B = !r.p || p == 0.0 ? 0.0 : 1.0 / p;
  f.mq = laws[(int64_t)b * (2 * K + 1) + r.iq].m;
  f.mp = r.p ? laws[(int64_t)b * (2 * K + 1) + r.ip].m : 0.f;
  if (f.mq == -INFINITY) f.mq = 0.f;
  if (f.mp == -INFINITY) f.mp = 0.f;
  return f;
}
// (two rounded products: equal laws differ by exactly 0.  One of them unrounded, in a fused
// operation, would leave the other's rounding, of which half is positive and would be drawn from.)
__device__ __forceinline__ double residual_weight(const Residual& f, float x, float y, Scale c) {
#pragma clang fp contract(off)
  const double q = f.A * weight(x, f.mq, c), p = f.B * weight(y, f.mp, c);
  const double w = q - p;
  return w > 0.0 ? w : 0.0;
}

// Vector k of this thread in a slice of both rows.
template <class T>
struct Two {
  Vec<T> x, y;
};
template <class T, int E>
__device__ __forceinline__ Two<T> load_two(const Pair<T>& r, bool with_p, int V, int slice, int k) {
  const int a = lead<T>(r.q);
  Two<T> v;
  v.x = load_vector<T, E>(r.q, a, V, slice, k);
  v.y = with_p ? load_vector<T, E>(r.p, a, V, slice, k) : v.x;
  return v;
}
// The residual's weights of such a pair; their sum.
template <class T>
__device__ __forceinline__ double residual_vector(const Residual& f, const Two<T>& v, bool with_p, Scale c,
                                                  double (&w)[T::kVec]) {
  double sum = 0.0;
  if (with_p) {
#pragma unroll
    for (int j = 0; j < T::kVec; ++j) sum += w[j] = residual_weight(f, T::value(v.x.r[j]), T::value(v.y.r[j]), c);
  } else {
#pragma unroll
    for (int j = 0; j < T::kVec; ++j) {
      const double g = f.A * weight(T::value(v.x.r[j]), f.mq, c);
      sum += w[j] = g > 0.0 ? g : 0.0;
    }
  }
  return sum;
}

// Slices of the residual's mass.  The workgroup of a chain that is done last finds the slice
// that the uniform falls into, and the token in it: the sums are read in the slices' order,
// so which one it is changes nothing.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void draw_token_kernel(
    Rows rows, int K, int V, int S, int mode, Scale c, const int32_t* __restrict__ kb,
    const int32_t* __restrict__ taus, const double* __restrict__ uniforms, const uint32_t* __restrict__ round,
    uint64_t seed, const Law* __restrict__ laws, const double* __restrict__ la, const Mass* __restrict__ sums,
    double* __restrict__ mass, uint32_t* __restrict__ arrived, int32_t* __restrict__ token) {
  constexpr int VEC = T::kVec, NV = E / VEC;
  __shared__ double red[4 * NV];
  __shared__ int ired[4];
  __shared__ double before_s;
  __shared__ int slice_s, tok_s, last_s;
  const int b = blockIdx.x / S, t = threadIdx.x;
  const int n = drafts(kb, b, K), tau = n > 0 ? taus[b] : 0;
  const Pair<T> r = drawn_rows<T>(rows, b, K, n, tau);
  if (!r.any) {
    if (blockIdx.x % S == 0 && t == 0) token[b] = -1;
    return;
  }
  Two<T> two = load_two<T, E>(r, r.p != nullptr, V, blockIdx.x % S, 0);
  const Residual f = residual_of<T>(r, b, K, S, mode, tau, laws, la, sums, red);
  double w[VEC];
  {
    double s = 0.0;
#pragma unroll 1
    for (int k = 0; k < NV; ++k) {
      const Two<T> next = k + 1 < NV ? load_two<T, E>(r, r.p != nullptr, V, blockIdx.x % S, k + 1) : two;
      s += residual_vector<T>(f, two, r.p != nullptr, c, w);
      two = next;
    }
    s = block_sum(s, red);
    if (t == 0) {
      // Atomics of device scope go past what the XCDs' caches may hold of their own, so a wait for
      // the store is all that orders it; a device-scope fence would write back the whole L2 here,
      // once a workgroup (64 chains of 131072 tokens: 75 us in all with the fence).
      __hip_atomic_store(&mass[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      last_s = __hip_atomic_fetch_add(&arrived[b], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)S - 1u;
    }
  }
  __syncthreads();
  if (!last_s) return;
  auto mass_of = [&](int s) {
    return __hip_atomic_load(&mass[(int64_t)b * S + s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };

  double u;
  if (uniforms) {
    u = uniforms[(int64_t)b * (K + 1) + K];
  } else {
    const uint4 x = philox(0u, (uint32_t)b, round[b], TAG_USAMPLE << 24, seed);
    u = ((double)(((uint64_t)(x.x >> 6) << 26) | (x.y >> 6)) + 0.5) * 0x1p-52;
  }
  // Laws without mass or with a NaN: the residual's sums come out 0 (a NaN weight
  // counts 0), the target's are then taken, and those decide.
  const int per = (S + kThreads - 1) / kThreads, s0 = min(t * per, S), s1 = min(s0 + per, S);
  double v = 0.0;
  for (int s = s0; s < s1; ++s) v += mass_of(s);
  double cum = block_scan(v, red);
  __syncthreads();
  if (t == kThreads - 1) before_s = cum;
  if (t == 0) {
    slice_s = -1;
    tok_s = -1;
  }
  __syncthreads();
  double all = before_s;
  const double qsum = f.A;  // 0 or NaN where the target has no law
  const bool use_q = !(all > 0.0);
  const bool nan = !(qsum > 0.0) || !isfinite(qsum) || (r.p && !isfinite(f.B));
  if (nan) {
    if (t == 0) token[b] = -1;
    return;
  }
  if (use_q) {
    v = 0.0;
    for (int s = s0; s < s1; ++s) v += sums[(int64_t)b * S + s].q * f.A;
    cum = block_scan(v, red);
    __syncthreads();
    if (t == kThreads - 1) before_s = cum;
    __syncthreads();
    all = before_s;
  }
  const double goal = u * all;
  // (a thread without mass is never chosen: added up in another order, its sum may exceed the one
  // before it, and the goal, by a bit)
  int owner = block_first(v > 0.0 && cum > goal, ired);
  if (owner == kThreads) owner = block_last(v > 0.0, ired);  // u next to 1
  if (owner < 0) {
    if (t == 0) token[b] = -1;
    return;
  }
  __syncthreads();
  if (t == owner) {
    double at = cum - v;
    int last = s0;
    for (int s = s0; s < s1; ++s) {
      const double g = use_q ? sums[(int64_t)b * S + s].q * f.A : mass_of(s);
      if (g > 0.0) {
        last = s;
        before_s = at;
        if (at + g > goal) break;
      }
      at += g;
    }
    slice_s = last;
  }
  __syncthreads();
  // the slice's weights again, in vectors of kThreads * VEC elements that follow one another
  const int slice = slice_s;
  const bool with_p = r.p && !use_q;
  double mine = 0.0;
  two = load_two<T, E>(r, with_p, V, slice, 0);
#pragma unroll 1
  for (int k = 0; k < NV; ++k) {
    const Two<T> next = k + 1 < NV ? load_two<T, E>(r, with_p, V, slice, k + 1) : two;
    mine = residual_vector<T>(f, two, with_p, c, w);
    two = next;
    const double s = wave_sum(mine);
    if ((t & 63) == 0) red[4 * k + (t >> 6)] = s;
  }
  __syncthreads();
  double before = before_s, upto = before;
  int vec = 0;
  bool past = false;
  for (int k = 0; k < NV; ++k) {
    const double g = red[4 * k] + red[4 * k + 1] + (red[4 * k + 2] + red[4 * k + 3]);
    if (!past && g > 0.0) {
      vec = k;
      before = upto;
      past = upto + g > goal;
    }
    upto += g;
  }
  if (vec != NV - 1) mine = residual_vector<T>(f, load_two<T, E>(r, with_p, V, slice, vec), with_p, c, w);
  __syncthreads();
  const double end = before + block_scan(mine, red);
  int who = block_first(mine > 0.0 && end > goal, ired);
  if (who == kThreads) who = block_last(mine > 0.0, ired);
  if (t == who) {
    double at = end - mine;
    int tok = -1;
    bool found = false;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      at += w[j];
      if (!found && w[j] > 0.0) {
        tok = position<T, E>(slice, lead<T>(r.q), vec * VEC + j);
        found = at > goal;
      }
    }
    tok_s = tok;
  }
  __syncthreads();
  if (t == 0) token[b] = tok_s;
}

// Short rows are each one workgroup's, in one kernel, where there is a compute unit for every
// one.  In us, two kernels / one: a row of 32000 float32, 20 alternatives, 14.1 / 9.0, bf16
// 11.5 / 7.4; 256 rows of 32000 bf16 15.7 / 9.8; 512 18.0 / 17.4, of 8000 16.1 / 18.0; 2048 of
// 32000 float32 44 / 67.  (Longer rows of 16 bits, 64 elements a thread: 11.9 + 6.2 / 27 for 256 of 65000.)
constexpr int kOneEach = 256;

template <class T, int E>
hipError_t logprobs_run(int rows, int V, const void* x, int64_t ld, double inv_t, int n_tok, const int32_t* tokens,
                        float* logprob, float* entropy, float* lse, int n, int32_t* ids, float* tops, void* ws,
                        hipStream_t s) {
  typedef typename T::raw raw;
  if (rows <= kOneEach && V + 7 <= kRowThreads * 32)
    return launch_timed("logprobs_row", logprobs_row_kernel<T, 32>, dim3((unsigned)rows), dim3(kRowThreads), s,
                        static_cast<const raw*>(x), ld, V, (float)(inv_t * kLog2e), inv_t, n_tok, tokens, logprob,
                        entropy, lse, n, ids, tops);
  const int S = slices(V, E);
  Part* parts = static_cast<Part*>(ws);
  uint64_t* keys = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + up256(sizeof(Part) * (size_t)rows * S));
  hipError_t e = launch_timed("logprobs_slice", logprobs_slice_kernel<T, E>, dim3((unsigned)((int64_t)rows * S)),
                              dim3(kThreads), s, static_cast<const raw*>(x), ld, V, S, (float)(inv_t * kLog2e), n,
                              parts, keys);
  if (e != hipSuccess) return e;
  return launch_timed("logprobs_join", logprobs_join_kernel<T>, dim3(rows), dim3(kThreads), s,
                      static_cast<const raw*>(x), ld, V, S, inv_t, n_tok, tokens, logprob, entropy, lse, n, ids, tops,
                      (const Part*)parts, (const uint64_t*)keys);
}

struct VerifyWs {
  size_t parts, laws, la, excess, sums, mass, arrived, bytes;
};
VerifyWs verify_layout(int B, int K, int V) {
  const int64_t rows = (int64_t)B * (2 * K + 1);
  const size_t S = (size_t)slices(V, per_thread(rows, V)), Sd = (size_t)slices(V, per_thread(B, V));
  VerifyWs w;
  w.parts = 0;
  w.laws = w.parts + up256(sizeof(Part) * (size_t)rows * S);
  w.la = w.laws + up256(sizeof(Law) * (size_t)rows);
  w.excess = w.la + up256(sizeof(double) * (size_t)B * K);
  w.sums = w.excess + up256(sizeof(double) * (size_t)B * K * S);
  w.mass = w.sums + up256(sizeof(Mass) * (size_t)B * Sd);
  w.arrived = w.mass + up256(sizeof(double) * (size_t)B * Sd);
  w.bytes = w.arrived + up256(sizeof(uint32_t) * (size_t)B);
  return w;
}

template <class T, int E>
hipError_t verify_run(const Rows& rows, int B, int K, int V, int mode, double inv_t, const int32_t* tokens,
                      const int32_t* kb, const double* uniforms, const uint32_t* round, uint64_t seed, int32_t* tau,
                      float* lar, float* ratio, uint64_t* coins, char* ws, const VerifyWs& w, hipStream_t s) {
  const int S = slices(V, E);
  const Scale c = scale_of(inv_t);
  Part* parts = reinterpret_cast<Part*>(ws + w.parts);
  Law* laws = reinterpret_cast<Law*>(ws + w.laws);
  double *la = reinterpret_cast<double*>(ws + w.la), *excess = reinterpret_cast<double*>(ws + w.excess);
  hipError_t e = launch_timed("verify_sums", verify_sums_kernel<T, E>, dim3((unsigned)((int64_t)B * (2 * K + 1) * S)),
                              dim3(kThreads), s, rows, K, V, S, c, kb, parts);
  if (e != hipSuccess) return e;
  e = launch_timed("verify_join", verify_join_kernel<T>, dim3(B), dim3(kThreads), s, rows, K, V, S, mode, inv_t,
                   tokens, kb, uniforms, round, seed, (const Part*)parts, laws, la, tau, lar, ratio, coins);
  if (e != hipSuccess || mode != SD_BLOCK || K == 1) return e;
  return launch_timed("verify_excess", verify_excess_kernel<T, E>, dim3((unsigned)((int64_t)B * (K - 1) * S)),
                      dim3(kThreads), s, rows, K, V, S, c, kb, (const Law*)laws, (const double*)la, excess);
}

// Se: the slices of a row in verify_run.
template <class T, int E>
hipError_t draw_run(const Rows& rows, int B, int K, int V, int Se, int mode, double inv_t, const int32_t* kb,
                    const double* uniforms, const uint32_t* round, uint64_t seed, int32_t* tau, int32_t* token,
                    float* lar, uint64_t* coins, char* ws, const VerifyWs& w, hipStream_t s) {
  const int S = slices(V, E);
  const Scale c = scale_of(inv_t);
  const Law* laws = reinterpret_cast<const Law*>(ws + w.laws);
  const double *la = reinterpret_cast<const double*>(ws + w.la),
               *excess = reinterpret_cast<const double*>(ws + w.excess);
  Mass* sums = reinterpret_cast<Mass*>(ws + w.sums);
  double* mass = reinterpret_cast<double*>(ws + w.mass);
  uint32_t* arrived = reinterpret_cast<uint32_t*>(ws + w.arrived);
  const dim3 grid((unsigned)((int64_t)B * S));
  hipError_t e = launch_timed("draw_sums", draw_sums_kernel<T, E>, grid, dim3(kThreads), s, rows, K, V, S, c, kb,
                              uniforms, round, seed, laws, la, mode == SD_BLOCK ? excess : nullptr, Se, tau, lar,
                              coins, sums, arrived);
  if (e != hipSuccess) return e;
  return launch_timed("draw_token", draw_token_kernel<T, E>, grid, dim3(kThreads), s, rows, K, V, S, mode, c, kb,
                      (const int32_t*)tau, uniforms, round, seed, laws, la, (const Mass*)sums, mass, arrived, token);
}

// Where each row is read for itself: eight vectors a thread instead of 32 elements, so that
// more elements share a slice's reductions.
template <class T>
int per_thread_alone(int64_t rows, int V) {
  return per_thread(rows, V) == 32 ? 8 * T::kVec : 8;
}

}  // namespace

size_t logprobs_ws_bytes(int rows, int V, int n) {
  const size_t S = (size_t)slices(V, per_thread(rows, V));  // (as many as any type has)
  return up256(sizeof(Part) * (size_t)rows * S) + up256(sizeof(uint64_t) * (size_t)rows * S * (size_t)n);
}
int64_t logprobs_groups(int rows, int V, sd_type type) {
  return (int64_t)rows * slices(V, by_type(type, [&](auto tag) { return per_thread_alone<decltype(tag)>(rows, V); }));
}

hipError_t logprobs_launch(int rows, int V, sd_type type, const void* x, int64_t ld, double temperature, int n_tok,
                           const int32_t* tokens, float* logprob, float* entropy, float* lse, int n, int32_t* ids,
                           float* tops, void* ws, hipStream_t s) {
  const double inv_t = 1.0 / temperature;
  return by_type(type, [&](auto tag) {
    typedef decltype(tag) T;
    return per_thread_alone<T>(rows, V) > 8
               ? logprobs_run<T, 8 * T::kVec>(rows, V, x, ld, inv_t, n_tok, tokens, logprob, entropy, lse, n, ids, tops, ws, s)
               : logprobs_run<T, 8>(rows, V, x, ld, inv_t, n_tok, tokens, logprob, entropy, lse, n, ids, tops, ws, s);
  });
}

size_t verify_tokens_ws_bytes(int B, int K, int V) { return verify_layout(B, K, V).bytes; }
int64_t verify_tokens_groups(int B, int K, int V) {
  const int64_t rows = (int64_t)B * (2 * K + 1);
  return rows * slices(V, per_thread(rows, V));
}

hipError_t verify_tokens_launch(int B, int K, int V, int mode, sd_type type, double temperature, const void* draft,
                                sd_stride ds, const void* target, sd_stride ts, const int32_t* tokens,
                                const int32_t* kb, const double* uniforms, const uint32_t* round, uint64_t seed,
                                int32_t* tau, int32_t* token, float* lar, float* ratio, uint64_t* coins, void* ws,
                                hipStream_t s) {
  const double inv_t = 1.0 / temperature;
  const Rows rows{draft, target, ds, ts};
  const VerifyWs w = verify_layout(B, K, V);
  char* base = static_cast<char*>(ws);
  return by_type(type, [&](auto tag) {
    typedef decltype(tag) T;
    hipError_t e = per_thread((int64_t)B * (2 * K + 1), V) == 32
                       ? verify_run<T, 32>(rows, B, K, V, mode, inv_t, tokens, kb, uniforms, round, seed, tau, lar,
                                           ratio, coins, base, w, s)
                       : verify_run<T, 8>(rows, B, K, V, mode, inv_t, tokens, kb, uniforms, round, seed, tau, lar,
                                          ratio, coins, base, w, s);
    if (e != hipSuccess) return e;
    const int Se = slices(V, per_thread((int64_t)B * (2 * K + 1), V));
    return per_thread(B, V) == 32 ? draw_run<T, 32>(rows, B, K, V, Se, mode, inv_t, kb, uniforms, round, seed, tau,
                                                    token, lar, coins, base, w, s)
                                  : draw_run<T, 8>(rows, B, K, V, Se, mode, inv_t, kb, uniforms, round, seed, tau,
                                                   token, lar, coins, base, w, s);
  });
}

}  // namespace sd
