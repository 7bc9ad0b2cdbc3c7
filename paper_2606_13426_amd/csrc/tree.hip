// Verification of trees of drafted tokens (gfx950): multi-round token verification along the
// branches, and the draw of the token that follows.
//
// A node's children are tries at one law q with a shared draft law p (laws.hpp).  After k
// rejected ones the rest is r_k = max(0, q - a_k p) / S_k with a_0 = 0, S_0 = 1,
//   S_k = sum max(0, q - a_k p),   a_{k+1} = a_k + S_k / rest_k:
// max(0, r_k - p / rest_k) has the positive part where q > (a_k + S_k / rest_k) p.  rest_k is 1
// for independent draws; for draws without replacement what the tries so far leave of p, summed
// beside S_k (1 less their mass is no number where p is all but one token), and a tried x
// needs no care in S_k: it was rejected, so q(x) < a_{k+1} p(x), and a only grows.  The k-th child is accepted with h_k = max(0, q/p - a_k) rest_k / S_k.  So a try behind the
// first costs one sum over the vocabulary.  Given candidates cost none: r_k is q without
// the tried ones, h_k = q(x) / (1 - their mass).
//
// Kernels: the trees (who has which children); both laws of every node with children, whose
// last workgroup tries the first child; a sum a round for the nodes that are
// undecided, whose last workgroup tries the next child; the draw, which walks the
// decided nodes from the root, sums the last r in slices and finds the token.  Nodes off the
// accepted branch are decided too: they are not known to be off it before.  All in
// float64, as every border is compared with a uniform.
#include "common.hpp"
#include "laws.hpp"
#include "logits.hpp"
#include "philox.hpp"
#include "wavered.hpp"

namespace sd {
namespace {

using namespace laws;

constexpr int kNodes = SD_MAX_TREE;
constexpr int kOpen = -2, kNone = -1;  // Node::next: not decided yet; no child accepted

struct Node {
  double Sq, Sp;  // the laws' sums against mq and mp: 0 for a row of -inf, NaN for no law
  double a, S;    // a_k, S_k
  double rest;    // rest_k; GIVEN: what the tried tokens leave of q
  uint64_t kids;  // children, bits
  float mq, mp;
  int32_t next, tried;  // the accepted child, kNone or kOpen; how many children were tried
};

struct Tree {
  Node* nodes;       // [B][Q]
  int32_t* list;     // [B][Q] nodes with children, rising
  int32_t* count;    // [B]
  uint32_t* arrived; // [B][Q + 1] workgroups that are done with a node, with the draw
  float* chance;     // [B][Q] min(1, h) of tried nodes
  double* sums;      // [B][Q][S][2] slices' sums of q and p, then of max(0, q - a p) and of p
  float* maxima;     // [B][Q][S][2]
  double* mass;      // [B][Sd][2] slices of the last r and of q
  float* peak;       // [B][Sd] the maximum that a slice's sums are against
};

template <class T>
__device__ __forceinline__ const typename T::raw* row_of(const void* p, sd_stride s, int b, int i) {
  return reinterpret_cast<const typename T::raw*>(p) + (int64_t)b * s.chain + (int64_t)i * s.row;
}
__device__ __forceinline__ int rows_of(const VerifyTreeArgs& a, int b) {
  return a.rows ? min(max(a.rows[b], 0), a.Q) : a.Q;
}

// Device-scope atomics go past what an XCD's caches hold of their own, so a wait for the store is all that
// orders it before the count.
__device__ __forceinline__ void put(double* p, double v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put(float* p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class V>
__device__ __forceinline__ V get(const V* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// One more workgroup is done; whether it is the last of `all`.
__device__ __forceinline__ bool last_of(uint32_t* arrived, uint32_t all) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  return __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1u;
}

// One wavefront a sequence: every node's children, the nodes that have some and that the root reaches.
__global__ __launch_bounds__(64) void tree_plan_kernel(VerifyTreeArgs a, Tree w) {
  const int b = blockIdx.x, lane = threadIdx.x, n = rows_of(a, b);
  int up = lane > 0 && lane < n ? a.parents[(int64_t)b * a.Q + lane] : -1;
  if (up < 0 || up >= lane) up = -1;
  uint64_t same = 0, kids = 0;  // nodes of this one's parent; this one's children
  for (int j = 1; j < n; ++j) {
    const int p = __builtin_amdgcn_readlane(up, j);
    if (p >= 0 && p == up) same |= 1ull << j;
    if (p == lane) kids |= 1ull << j;
  }
  // children past max_children are no part of the tree
  if (__popcll(same & ((1ull << lane) - 1ull)) >= a.max_children) up = -1;
  uint64_t left = kids;
  for (int k = 0; k < a.max_children && left; ++k) left &= left - 1;
  kids &= ~left;
  bool reached = lane == 0;
  for (int j = 1; j < n; ++j) {  // (a parent comes before its children)
    const uint64_t so_far = __ballot(reached);
    const int p = __builtin_amdgcn_readlane(up, j);
    if (lane == j && p >= 0 && (so_far >> p & 1u)) reached = true;
  }
  const uint64_t inner = __ballot(lane < n && reached && kids != 0);
  if (inner >> lane & 1u) w.list[(int64_t)b * a.Q + __popcll(inner & ((1ull << lane) - 1ull))] = lane;
  if (lane == 0) w.count[b] = __popcll(inner);
  if (lane < a.Q) {
    Node v{};
    v.kids = kids;
    v.S = v.rest = 1.0;
    v.next = kids ? kOpen : kNone;
    w.nodes[(int64_t)b * a.Q + lane] = v;
    w.arrived[(int64_t)b * (a.Q + 1) + lane] = 0;
    w.chance[(int64_t)b * a.Q + lane] = -1.f;
  }
  if (lane == 0) w.arrived[(int64_t)b * (a.Q + 1) + a.Q] = 0;
}

// Coin of node i >= 1, and the draw's uniform.
__device__ __forceinline__ double eta_of(const VerifyTreeArgs& a, int b, int i) {
  if (a.uniforms) return a.uniforms[(int64_t)b * a.Q + i - 1];
  const uint4 x = philox((uint32_t)((i - 1) >> 2), (uint32_t)b, a.round[b], TAG_COIN << 24, a.seed);
  return uniform64(pick(x, (i - 1) & 3));
}
__device__ __forceinline__ double draw_of(const VerifyTreeArgs& a, int b) {
  if (a.uniforms) return a.uniforms[(int64_t)b * a.Q + a.Q - 1];
  const uint4 x = philox(0u, (uint32_t)b, a.round[b], TAG_USAMPLE << 24, a.seed);
  return ((double)(((uint64_t)(x.x >> 6) << 26) | (x.y >> 6)) + 0.5) * 0x1p-52;
}

// The tries of node i that need no further sum, by one wavefront; v is its state, S_k in it.
template <class T>
__device__ __forceinline__ void tries(const VerifyTreeArgs& a, const Tree& w, int b, int i, Node v, double inv_t) {
  const int lane = threadIdx.x & 63;
  const bool mine = v.kids >> lane & 1u;
  // every child's token, coin, log-ratio and draft probability, a lane each
  const int x = mine ? a.tokens[(int64_t)b * a.Q + lane] : -1;
  const bool known = x >= 0 && x < a.V;
  const float xq = known ? T::value(row_of<T>(a.target, a.ts, b, i)[x]) : -INFINITY;
  const float xp = known && a.draft ? T::value(row_of<T>(a.draft, a.ds, b, i)[x]) : -INFINITY;
  const double eta = mine ? eta_of(a, b, lane) : 2.0;
  const bool okq = v.Sq >= 0.0 && isfinite(v.Sq), okp = a.draws == SD_TREE_GIVEN || (v.Sp >= 0.0 && isfinite(v.Sp));
  // (a log-ratio below 2^-44 is one of sums added in another order: 0)
  double ratio = 0.0, q = 0.0;  // q / p, q
  if (known && okq && okp && v.Sq > 0.0 && xq > -INFINITY) {
    const double zq = ((double)xq - (double)v.mq) * inv_t;
    q = exp(zq) / v.Sq;
    if (a.draws == SD_TREE_GIVEN) {
      // (the candidate's own law is all on it)
    } else if (v.Sp == 0.0 || xp == -INFINITY) {
      ratio = INFINITY;
    } else {
      const double ell = zq - ((double)xp - (double)v.mp) * inv_t - (log(v.Sq) - log(v.Sp));
      ratio = fabs(ell) < 0x1p-44 ? 1.0 : exp(ell);
    }
  }
  uint64_t left = v.kids;
  for (int k = 0; k < v.tried; ++k) left &= left - 1;
  float chance = -1.f;
  v.next = kOpen;
  while (left) {
    const int j = __ffsll((unsigned long long)left) - 1;
    left &= left - 1;
    ++v.tried;
    const int tok = __shfl(x, j);
    const bool valid = __shfl((int)known, j) != 0 && okq && okp;
    const bool again = __ballot(mine && lane < j && x == tok) != 0;
    const double qj = __shfl(q, j), rj = __shfl(ratio, j), coin = __shfl(eta, j);
    double h = 0.0;
    bool spent = false;  // a try that the next ones' law knows of
    if (valid && (a.draws == SD_TREE_IID || !again)) {
      if (a.draws == SD_TREE_GIVEN) {
        // (by a difference: a rest as small as its rounding is reached as seldom)
        h = qj > 0.0 ? qj / fmax(v.rest, qj) : 0.0;
        v.rest -= qj;
      } else {
        const double over = fmax(rj - v.a, 0.0);
        spent = v.rest > 0.0;  // (else a draw of what is nothing in float64: as one of draft probability 0)
        h = !(over > 0.0 && v.S > 0.0) ? 0.0
            : !spent               ? (qj > 0.0 ? 1.0 : 0.0)
            : rj == (double)INFINITY ? 1.0 : over * v.rest / v.S;
        if (coin >= h && spent) v.a += v.S / v.rest;
      }
    }
    if (lane == j) chance = (float)fmin(h, 1.0);
    if (coin < h) {
      v.next = j;
      break;
    }
    if (spent && left) break;  // the next try needs S of the new a
  }
  if (v.next == kOpen && !left) v.next = kNone;
  if (chance >= 0.f) w.chance[(int64_t)b * a.Q + lane] = chance;
  if (lane == 0) w.nodes[(int64_t)b * a.Q + i] = v;
}

// Node r of the list of sequence b, or -1.
__device__ __forceinline__ int listed(const VerifyTreeArgs& a, const Tree& w, int b, int r) {
  return r < w.count[b] ? w.list[(int64_t)b * a.Q + r] : -1;
}

// Slices of both laws' sums of a node with children.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void tree_sums_kernel(VerifyTreeArgs a, Tree w, int S, int R, Scale c, double inv_t) {
  __shared__ double red[4], joined[2];
  __shared__ float redm[4], peaks[2];
  __shared__ int last_s;
  const int slice = blockIdx.x % S, t = threadIdx.x;
  const int64_t id = blockIdx.x / S;
  const int b = (int)(id / R);
  for (int r = (int)(id % R); r < a.Q; r += R) {
    const int i = listed(a, w, b, r);
    if (i < 0) return;
    const typename T::raw* pq = row_of<T>(a.target, a.ts, b, i);
    const typename T::raw* pp = a.draft ? row_of<T>(a.draft, a.ds, b, i) : nullptr;
    const int lead_q = lead<T>(pq);
    // (both rows by the target's vectors: equal rows have equal sums)
    float x[E], y[E];
    load_slice<T, E>(pq, lead_q, a.V, slice, x);
    if (pp) load_slice<T, E>(pp, lead_q, a.V, slice, y);
    const Part q = slice_sums64<T, E>(x, c, red, redm);
    __syncthreads();
    Part p{0.0, 0.0, -INFINITY, 0.f};
    if (pp) p = slice_sums64<T, E>(y, c, red, redm);
    const int64_t at = ((int64_t)b * a.Q + i) * S;
    if (t == 0) {
      put(&w.sums[2 * (at + slice)], q.S);
      put(&w.sums[2 * (at + slice) + 1], p.S);
      put(&w.maxima[2 * (at + slice)], q.m);
      put(&w.maxima[2 * (at + slice) + 1], p.m);
      last_s = last_of(&w.arrived[(int64_t)b * (a.Q + 1) + i], (uint32_t)S);
    }
    __syncthreads();
    if (last_s) {
      // the first wavefront joins q's slices, the second p's
      const int h = t >> 6, lane = t & 63;
      if (h < 2) {
        float m = -INFINITY;
        for (int s = lane; s < S; s += 64) m = fmaxf(m, get(&w.maxima[2 * (at + s) + h]));
        m = wave_max(m);
        double sum = 0.0;
        for (int s = lane; s < S; s += 64) {
          const float ms = get(&w.maxima[2 * (at + s) + h]);
          const double v = get(&w.sums[2 * (at + s) + h]);
          if (!(ms == -INFINITY && v == 0.0)) sum += v * exp(((double)ms - (double)m) * inv_t);
        }
        sum = wave_sum(sum);
        if (lane == 0) {
          joined[h] = sum;
          peaks[h] = m;
        }
      }
      __syncthreads();
      if (t < 64) {
        Node v = w.nodes[(int64_t)b * a.Q + i];
        v.Sq = joined[0];
        v.Sp = joined[1];
        v.mq = peaks[0] == -INFINITY ? 0.f : peaks[0];
        v.mp = peaks[1] == -INFINITY ? 0.f : peaks[1];
        tries<T>(a, w, b, i, v, inv_t);
      }
    }
    __syncthreads();
  }
}

// Slices of S_k of the nodes that need it for their next child; round k >= 1.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void tree_round_kernel(VerifyTreeArgs a, Tree w, int S, int R, int k, Scale c, double inv_t) {
  __shared__ double red[8];
  __shared__ int last_s;
  const int slice = blockIdx.x % S, t = threadIdx.x;
  const int64_t id = blockIdx.x / S;
  const int b = (int)(id / R);
  for (int r = (int)(id % R); r < a.Q; r += R) {
    const int i = listed(a, w, b, r);
    if (i < 0) return;
    const Node v = w.nodes[(int64_t)b * a.Q + i];
    if (v.next != kOpen) continue;
    const typename T::raw *pq = row_of<T>(a.target, a.ts, b, i), *pp = row_of<T>(a.draft, a.ds, b, i);
    const double A = v.Sq == 0.0 ? 0.0 : 1.0 / v.Sq, B = v.Sp == 0.0 ? 0.0 : v.a / v.Sp;
    const int lead_q = lead<T>(pq);
    float x[E], y[E];
    load_slice<T, E>(pq, lead_q, a.V, slice, x);
    load_slice<T, E>(pp, lead_q, a.V, slice, y);
    const bool distinct = a.draws == SD_TREE_DISTINCT;
    if (distinct) {
      // the tried tokens are out of p's sum, and have no part in the other
      uint64_t left = v.kids;
      for (int j = 0; j < v.tried; ++j, left &= left - 1) {
        const int tok = a.tokens[(int64_t)b * a.Q + __ffsll((unsigned long long)left) - 1];
        const int at = tok + lead_q, vec = at / T::kVec - slice * (E / T::kVec) * kThreads;
        if (tok < 0 || tok >= a.V || vec < 0 || vec % kThreads != t || vec / kThreads >= E / T::kVec) continue;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e == vec / kThreads * T::kVec + at % T::kVec) x[e] = y[e] = -INFINITY;
      }
    }
    double s[2] = {0.0, 0.0}, rest = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double wp = weight_or_tiny(y[e], v.mp, c);
      s[e & 1] += excess_of(A, weight_or_tiny(x[e], v.mq, c), B, wp);
      if (distinct) rest += wp;
    }
    const double sum = wave_sum(s[0] + s[1]);
    rest = wave_sum(rest);
    if ((t & 63) == 0) {
      red[t >> 6] = sum;
      red[4 + (t >> 6)] = rest;
    }
    __syncthreads();
    const int64_t at = ((int64_t)b * a.Q + i) * S;
    if (t == 0) {
      put(&w.sums[2 * (at + slice)], red[0] + red[1] + (red[2] + red[3]));
      put(&w.sums[2 * (at + slice) + 1], red[4] + red[5] + (red[6] + red[7]));
      last_s = last_of(&w.arrived[(int64_t)b * (a.Q + 1) + i], (uint32_t)(k + 1) * (uint32_t)S);
    }
    __syncthreads();
    if (last_s && t < 64) {
      double sum = 0.0, rest = 0.0;
      for (int j = t; j < S; j += 64) {
        sum += get(&w.sums[2 * (at + j)]);
        rest += get(&w.sums[2 * (at + j) + 1]);
      }
      Node u = v;
      u.S = wave_sum(sum);
      rest = wave_sum(rest);
      // (weights below 2^-1000 are 0, for which the sum has 2^-1000)
      if (distinct) u.rest = v.Sp > 0.0 && rest > 0x1p-960 ? rest / v.Sp : 0.0;
      tries<T>(a, w, b, i, u, inv_t);
    }
    __syncthreads();
  }
}

// The weight of an element of the last r: max(0, A wq - B wp), or A wq.
template <class T>
struct Drawn {
  const typename T::raw *q, *p;  // p: null where nothing is subtracted
  double A, B;
  float mq, mp;
};
// Vector k of this thread in a slice: its weights, wq without p's part, and their sums.
template <class T, int E>
__device__ __forceinline__ double drawn_vector(const Drawn<T>& d, const Vec<T>& x, const Vec<T>& y, bool with_p, Scale c,
                                               double (&w)[T::kVec], double& whole) {
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < T::kVec; ++j) {
    const double wq = weight(T::value(x.r[j]), d.mq, c), q = d.A * wq;
    whole += q;
    w[j] = with_p ? excess_of(d.A, wq, d.B, weight(T::value(y.r[j]), d.mp, c)) : q;
    sum += w[j];
  }
  return sum;
}

// Slices of the last r's mass.  The workgroup of a sequence that is done last finds the slice
// that the uniform falls into, and the token in it; the sums are read in the slices' order.  A node
// without children has no law yet: its slices are against their own maxima.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void tree_draw_kernel(VerifyTreeArgs a, Tree w, int S, Scale c, double inv_t) {
  constexpr int VEC = T::kVec, NV = E / VEC;
  __shared__ double red[4 * NV];
  __shared__ float redm[4];
  __shared__ int ired[4];
  __shared__ double before_s, goal_s;
  __shared__ int slice_s, tok_s, last_s, leaf_s;
  __shared__ int32_t gone[kNodes];  // GIVEN: the tokens that were tried below the last node
  __shared__ int gone_n;
  const int slice = blockIdx.x % S, b = blockIdx.x / S, t = threadIdx.x, n = rows_of(a, b);
  if (n == 0) {
    if (slice == 0) {
      if (t == 0) {
        a.tau[b] = 0;
        a.token[b] = -1;
      }
      if (t < a.Q) {
        a.path[(int64_t)b * a.Q + t] = -1;
        if (a.accept) a.accept[(int64_t)b * a.Q + t] = -1.f;
      }
    }
    return;
  }
  if (t < 64) {
    // the walk, by one wavefront: a lane holds a node
    const Node* nodes = w.nodes + (int64_t)b * a.Q;
    const int next = t < n ? nodes[t].next : kNone;
    const uint64_t kids = t < n ? nodes[t].kids : 0;
    int at = 0, steps = 1, mine = t == 0 ? 0 : -1;
    uint64_t seen = 0;  // children of the nodes that were passed
    for (;; ++steps) {
      const uint64_t of = (uint64_t)__shfl((unsigned long long)kids, at);
      const int to = __builtin_amdgcn_readlane(next, at);
      seen |= to >= 0 ? of & ((2ull << to) - 1ull) : of;
      if (to <= at) break;
      at = to;
      if (t == steps) mine = at;
    }
    if (slice == 0) {
      if (t == 0) a.tau[b] = steps;
      if (t < a.Q) {
        a.path[(int64_t)b * a.Q + t] = mine;
        if (a.accept) a.accept[(int64_t)b * a.Q + t] = seen >> t & 1u ? w.chance[(int64_t)b * a.Q + t] : -1.f;
      }
    }
    const uint64_t of = (uint64_t)__shfl((unsigned long long)kids, at);
    if (a.draws == SD_TREE_GIVEN && (of >> t & 1u)) gone[__popcll(of & ((1ull << t) - 1ull))] = a.tokens[(int64_t)b * a.Q + t];
    if (t == 0) {
      leaf_s = at;
      gone_n = a.draws == SD_TREE_GIVEN ? __popcll(of) : 0;
    }
  }
  __syncthreads();
  const int f = leaf_s;
  const Node v = w.nodes[(int64_t)b * a.Q + f];
  const bool inner = v.kids != 0;
  Drawn<T> d;
  d.q = row_of<T>(a.target, a.ts, b, f);
  d.p = inner && a.draft && v.a > 0.0 ? row_of<T>(a.draft, a.ds, b, f) : nullptr;
  d.A = !inner ? 1.0 : v.Sq == 0.0 ? 0.0 : 1.0 / v.Sq;
  d.B = d.p && v.Sp != 0.0 ? v.a / v.Sp : 0.0;
  d.mq = v.mq;
  d.mp = v.mp;
  const bool no_law = inner && (!(v.Sq > 0.0) || !isfinite(v.Sq) || (a.draft && !isfinite(v.Sp)));
  if (no_law) {
    if (slice == 0 && t == 0) a.token[b] = -1;
    return;
  }
  const int lead_q = lead<T>(d.q);
  // elements of vector k in slice s that were tried have no part in r
  auto without = [&](Vec<T>& x, int s, int k) {
    for (int j = 0; j < gone_n; ++j) {
      const int tok = gone[j], e = tok - position<T, E>(s, lead_q, k * VEC);
#pragma unroll
      for (int l = 0; l < VEC; ++l)
        if (tok >= 0 && e == l) x.r[l] = T::kNone;
    }
  };
  {
    Vec<T> x[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) x[k] = load_vector<T, E>(d.q, lead_q, a.V, slice, k);
    if (!inner) {
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = fmaxf(m, T::value(x[k].r[j]));
      m = wave_max(m);
      if ((t & 63) == 0) redm[t >> 6] = m;
      __syncthreads();
      m = fmaxf(fmaxf(redm[0], redm[1]), fmaxf(redm[2], redm[3]));
      d.mq = m == -INFINITY ? 0.f : m;
    }
    double s = 0.0, whole = 0.0, weights[VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Vec<T> y = d.p ? load_vector<T, E>(d.p, lead_q, a.V, slice, k) : x[k];
      if (gone_n) {
        Vec<T> all = x[k];
        double none = 0.0;
        drawn_vector<T, E>(d, all, all, false, c, weights, whole);
        without(all, slice, k);
        s += drawn_vector<T, E>(d, all, all, false, c, weights, none);
      } else {
        s += drawn_vector<T, E>(d, x[k], y, d.p != nullptr, c, weights, whole);
      }
    }
    if (!inner && d.mq == INFINITY) whole = NAN;
    s = block_sum(s, red);
    whole = block_sum(whole, red);
    if (t == 0) {
      const int64_t at = (int64_t)b * S + slice;
      put(&w.mass[2 * at], whole != whole ? NAN : s);
      put(&w.mass[2 * at + 1], whole);
      put(&w.peak[at], d.mq);
      last_s = last_of(&w.arrived[(int64_t)b * (a.Q + 1) + a.Q], (uint32_t)S);
    }
  }
  __syncthreads();
  if (!last_s) return;
  // the slices' masses against one maximum, a range of them a thread
  const int per = (S + kThreads - 1) / kThreads, s0 = min(t * per, S), s1 = min(s0 + per, S);
  const int64_t base = (int64_t)b * S;
  float m = -INFINITY;
  if (!inner) {
    for (int s = s0; s < s1; ++s)
      if (get(&w.mass[2 * (base + s) + 1]) != 0.0) m = fmaxf(m, get(&w.peak[base + s]));
    m = wave_max(m);
    if ((t & 63) == 0) redm[t >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(redm[0], redm[1]), fmaxf(redm[2], redm[3]));
  }
  auto factor = [&](int s) {
    if (inner) return 1.0;
    const double z = ((double)get(&w.peak[base + s]) - (double)m) * inv_t;
    return z < -700.0 ? 0.0 : exp(z);
  };
  bool use_q = false;
  auto mass_of = [&](int s) {
    const double g = get(&w.mass[2 * (base + s) + (use_q ? 1 : 0)]);
    return g == 0.0 ? 0.0 : g * factor(s);  // (a slice of -inf alone has no maximum)
  };
  double mass = 0.0, cum = 0.0, all = 0.0;
  auto total = [&] {
    mass = 0.0;
    for (int s = s0; s < s1; ++s) mass += mass_of(s);
    cum = block_scan(mass, red);
    __syncthreads();
    if (t == kThreads - 1) before_s = cum;
    __syncthreads();
    all = before_s;
  };
  total();
  if (!(all > 0.0) && all == all) {  // (nothing left of the last r: the target's own law)
    use_q = true;
    total();
  }
  if (!(all > 0.0) || !isfinite(all)) {
    if (t == 0) a.token[b] = -1;
    return;
  }
  const double goal = draw_of(a, b) * all;
  // (a thread without mass is never chosen: added up in another order, its sum may exceed the one
  // before it, and the goal, by a bit)
  int owner = block_first(mass > 0.0 && cum > goal, ired);
  if (owner == kThreads) owner = block_last(mass > 0.0, ired);  // u next to 1
  __syncthreads();
  if (t == owner) {
    double at = cum - mass;
    for (int s = s0; s < s1; ++s) {
      const double g = mass_of(s);
      if (g > 0.0) {
        slice_s = s;
        before_s = at;
        if (at + g > goal) break;
      }
      at += g;
    }
    // the rest of the way in the slice's own measure
    goal_s = (goal - before_s) / factor(slice_s);
  }
  if (t == 0) tok_s = -1;
  __syncthreads();
  const int found = slice_s;
  const double rest = goal_s;
  const bool with_p = d.p && !use_q;
  if (!inner) d.mq = get(&w.peak[base + found]);
  double weights[VEC], mine = 0.0, none = 0.0;
  auto vector = [&](int k) {
    Vec<T> x = load_vector<T, E>(d.q, lead_q, a.V, found, k);
    const Vec<T> y = with_p ? load_vector<T, E>(d.p, lead_q, a.V, found, k) : x;
    if (gone_n && !use_q) without(x, found, k);
    return drawn_vector<T, E>(d, x, y, with_p, c, weights, none);
  };
  for (int k = 0; k < NV; ++k) {
    const double s = wave_sum(vector(k));
    if ((t & 63) == 0) red[4 * k + (t >> 6)] = s;
  }
  __syncthreads();
  double before = 0.0, upto = 0.0;
  int vec = 0;
  bool past = false;
  for (int k = 0; k < NV; ++k) {
    const double g = red[4 * k] + red[4 * k + 1] + (red[4 * k + 2] + red[4 * k + 3]);
    if (!past && g > 0.0) {
      vec = k;
      before = upto;
      past = upto + g > rest;
    }
    upto += g;
  }
  mine = vector(vec);
  __syncthreads();
  const double end = before + block_scan(mine, red);
  int who = block_first(mine > 0.0 && end > rest, ired);
  if (who == kThreads) who = block_last(mine > 0.0, ired);
  if (t == who) {
    double at = end - mine;
    int tok = -1;
    bool there = false;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      at += weights[j];
      if (!there && weights[j] > 0.0) {
        tok = position<T, E>(found, lead_q, vec * VEC + j);
        there = at > rest;
      }
    }
    tok_s = tok;
  }
  __syncthreads();
  if (t == 0) a.token[b] = tok_s;
}

// Workgroups share a tree's nodes with children, of which branching trees have few: half as many as nodes
// take all of them, in two turns where the tree is a chain.
inline int workers(int Q) { return Q > 1 ? Q / 2 : 1; }
inline int64_t law_rows(int B, int Q) { return (int64_t)B * workers(Q); }

struct TreeWs {
  size_t nodes, list, count, arrived, chance, sums, maxima, mass, peak, bytes;
};
TreeWs tree_layout(int B, int Q, int V) {
  const size_t S = (size_t)slices(V, per_thread(law_rows(B, Q), V)), Sd = (size_t)slices(V, per_thread(B, V));
  const size_t n = (size_t)B * Q;
  TreeWs w;
  w.nodes = 0;
  w.list = w.nodes + up256(sizeof(Node) * n);
  w.count = w.list + up256(sizeof(int32_t) * n);
  w.arrived = w.count + up256(sizeof(int32_t) * (size_t)B);
  w.chance = w.arrived + up256(sizeof(uint32_t) * (n + B));
  w.sums = w.chance + up256(sizeof(float) * n);
  w.maxima = w.sums + up256(2 * sizeof(double) * n * S);
  w.mass = w.maxima + up256(2 * sizeof(float) * n * S);
  w.peak = w.mass + up256(2 * sizeof(double) * (size_t)B * Sd);
  w.bytes = w.peak + up256(sizeof(float) * (size_t)B * Sd);
  return w;
}

template <class T, int E>
hipError_t laws_run(const VerifyTreeArgs& a, const Tree& w, double inv_t, hipStream_t s) {
  const int S = slices(a.V, E), R = workers(a.Q);
  const Scale c = scale_of(inv_t);
  const dim3 grid((unsigned)((int64_t)a.B * R * S));
  hipError_t e = launch_timed("tree_sums", tree_sums_kernel<T, E>, grid, dim3(kThreads), s, a, w, S, R, c, inv_t);
  if (a.draws == SD_TREE_GIVEN) return e;
  for (int k = 1; k < a.max_children && k < a.Q - 1 && e == hipSuccess; ++k)
    e = launch_timed("tree_round", tree_round_kernel<T, E>, grid, dim3(kThreads), s, a, w, S, R, k, c, inv_t);
  return e;
}
template <class T, int E>
hipError_t draw_run(const VerifyTreeArgs& a, const Tree& w, double inv_t, hipStream_t s) {
  const int S = slices(a.V, E);
  return launch_timed("tree_draw", tree_draw_kernel<T, E>, dim3((unsigned)((int64_t)a.B * S)), dim3(kThreads), s, a, w,
                      S, scale_of(inv_t), inv_t);
}

}  // namespace

size_t verify_tree_ws_bytes(int B, int Q, int V) { return tree_layout(B, Q, V).bytes; }
int64_t verify_tree_groups(int B, int Q, int V) {
  const int64_t laws = law_rows(B, Q) * slices(V, per_thread(law_rows(B, Q), V));
  return laws > (int64_t)B * slices(V, per_thread(B, V)) ? laws : (int64_t)B * slices(V, per_thread(B, V));
}

hipError_t verify_tree_launch(const VerifyTreeArgs& a, sd_type type, double temperature, void* ws, hipStream_t s) {
  const double inv_t = 1.0 / temperature;
  const TreeWs l = tree_layout(a.B, a.Q, a.V);
  char* base = static_cast<char*>(ws);
  const Tree w{reinterpret_cast<Node*>(base + l.nodes),       reinterpret_cast<int32_t*>(base + l.list),
               reinterpret_cast<int32_t*>(base + l.count),    reinterpret_cast<uint32_t*>(base + l.arrived),
               reinterpret_cast<float*>(base + l.chance),     reinterpret_cast<double*>(base + l.sums),
               reinterpret_cast<float*>(base + l.maxima),     reinterpret_cast<double*>(base + l.mass),
               reinterpret_cast<float*>(base + l.peak)};
  hipError_t e = launch_timed("tree_plan", tree_plan_kernel, dim3((unsigned)a.B), dim3(64), s, a, w);
  if (e != hipSuccess) return e;
  return by_type(type, [&](auto tag) {
    typedef decltype(tag) T;
    hipError_t e = hipSuccess;
    if (a.Q > 1) e = per_thread(law_rows(a.B, a.Q), a.V) == 32 ? laws_run<T, 32>(a, w, inv_t, s) : laws_run<T, 8>(a, w, inv_t, s);
    if (e != hipSuccess) return e;
    return per_thread(a.B, a.V) == 32 ? draw_run<T, 32>(a, w, inv_t, s) : draw_run<T, 8>(a, w, inv_t, s);
  });
}

}  // namespace sd
