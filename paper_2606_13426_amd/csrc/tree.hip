// Verification of trees of drafted tokens (gfx950): multi-round token verification along the
// branches, and the draw of the token that follows.
//
// A node's children are tries at one law q with a shared draft law p (laws.hpp).  After k
// rejected ones the rest is r_k = max(0, q - a_k p) / S_k with a_0 = 0, S_0 = 1,
//   S_k = sum max(0, q - a_k p),   a_{k+1} = a_k + S_k / rest_k:
// max(0, r_k - p / rest_k) has the positive part where q > (a_k + S_k / rest_k) p.  rest_k is 1
// for independent draws; for draws without replacement what the tries so far leave of p, summed
// beside S_k (1 less their mass is no number where p is all but one token), and a tried x
// needs no care in S_k: it was rejected, so q(x) < a_{k+1} p(x), and a only grows.  The k-th
// child is accepted with h_k = max(0, q/p - a_k) rest_k / S_k.  So a try behind the first costs
// one sum over the vocabulary.  Given candidates cost none: r_k is q without the tried
// ones, h_k = q(x) / (1 - their mass).
//
// Kernels: the trees (who has which children); steps, each of which makes the next sum of every open
// node that the walk may still come to (both laws, then S_k), slices of a row a workgroup, and the last of
// a node's workgroups does the tries that the sum allows; the draw, which walks the decided
// nodes from the root, sums the last r in slices and finds the token.  How many steps there are is
// known on the host: one for the laws (three and more where they are much work) and one for every child behind
// the first, and a node that is out by then costs nothing.  All in float64, as every border is
// compared with a uniform.
//
// What bounds it: float64 exponentials, 16 products each (1.2e12 a second reached), where laws are summed, and for
// small calls launches and each one's trips to memory (3 to 6 us for the trees, 4 to 14 a later step, 10 to 20 the draw).  In
// us, a call among others / in a graph of its own: 1 tree of 12 over 32000 28 to 30 / 36, 24 of 24 over 50001 (given) 41 /
// 44, 32 of 32 over 131072 (distinct) 144 to 155 / 139 (190 with every node's laws at once).
#include "common.hpp"
#include "laws.hpp"
#include "logits.hpp"
#include "philox.hpp"
#include "wavered.hpp"

namespace sd {
namespace {

using namespace laws;

constexpr int kNodes = SD_MAX_TREE;
constexpr int kOpen = 0, kNone = 1;  // Node::state: not decided yet; no child accepted; the accepted child + 1

struct Node {
  double Sq, Sp;  // the laws' sums against mq and mp: 0 for a row of -inf, NaN for no law
  double a, S;    // a_k, S_k
  double rest;    // rest_k; GIVEN: what the tried tokens leave of q
  uint64_t kids;  // children, bits
  float mq, mp;
  int32_t state;  // in one word, as others read it while it changes: the decision, 256 times the children tried
  int32_t steps;  // sums that were made for it
};
__device__ __forceinline__ int decided(int state) { return state & 255; }

struct Tree {
  Node* nodes;       // [B][Q]
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
__device__ __forceinline__ void put(uint32_t* p, uint32_t v) {
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
  if (!reached) kids = 0;
  if (lane < a.Q) {
    Node v{};
    v.kids = kids;
    v.S = v.rest = 1.0;
    v.state = kids ? kOpen : kNone;
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

// What a child brings to its try, a lane each: its token, the logits there, its coin.
struct Child {
  double eta;
  int x;
  bool known;
  float xq, xp;
};
template <class T>
__device__ __forceinline__ Child child_of(const VerifyTreeArgs& a, int b, int i, uint64_t kids) {
  const int lane = threadIdx.x & 63;
  const bool mine = kids >> lane & 1u;
  Child k;
  k.x = mine ? a.tokens[(int64_t)b * a.Q + lane] : -1;
  k.eta = mine ? eta_of(a, b, lane) : 2.0;
  k.known = k.x >= 0 && k.x < a.V;
  k.xq = k.known ? T::value(row_of<T>(a.target, a.ts, b, i)[k.x]) : -INFINITY;
  k.xp = k.known && a.draft ? T::value(row_of<T>(a.draft, a.ds, b, i)[k.x]) : -INFINITY;
  return k;
}

// The tries of node i that need no further sum, by one wavefront; v is its state, S_k in it.
__device__ __forceinline__ void tries(const VerifyTreeArgs& a, const Tree& w, int b, int i, Node v, const Child& child, double inv_t) {
  const int lane = threadIdx.x & 63, x = child.x;
  const bool mine = v.kids >> lane & 1u, known = child.known;
  const float xq = child.xq, xp = child.xp;
  const double eta = child.eta;
  // every child's log-ratio and draft probability
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
  int tried = v.state >> 8, next = kOpen;
  uint64_t left = v.kids;
  for (int k = 0; k < tried; ++k) left &= left - 1;
  float chance = -1.f;
  while (left) {
    const int j = __ffsll((unsigned long long)left) - 1;
    left &= left - 1;
    ++tried;
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
      next = j + 1;
      break;
    }
    if (spent && left) break;  // the next try needs S of the new a
  }
  if (next == kOpen && !left) next = kNone;
  v.state = tried << 8 | next;
  ++v.steps;
  if (chance >= 0.f) w.chance[(int64_t)b * a.Q + lane] = chance;
  if (lane == 0) w.nodes[(int64_t)b * a.Q + i] = v;
}

enum { kLaws = 1, kExcess = 2, kBoth = 3 };
// One sum of a node, the next that it needs: of both laws, or S_k (SUMS: the ones that there may be).  Its workgroups hold a slice each, and
// the one that is done last goes on to the tries that the sum allows.
template <class T, int E, int SUMS>
__device__ __forceinline__ void node_step(const VerifyTreeArgs& a, const Tree& w, int b, int i, const Node& v, int slice, int S,
                                          Scale c, double inv_t) {
  __shared__ double red[8], joined[2];
  __shared__ float redm[4], peaks[2];
  __shared__ int last_s;
  const int t = threadIdx.x;
  const bool first = SUMS == kLaws || (SUMS == kBoth && v.steps == 0), distinct = a.draws == SD_TREE_DISTINCT;
  const typename T::raw* pq = row_of<T>(a.target, a.ts, b, i);
  const typename T::raw* pp = a.draft ? row_of<T>(a.draft, a.ds, b, i) : nullptr;
  const int lead_q = lead<T>(pq);
  // (both rows by the target's vectors: equal rows have equal sums)
  float x[E], y[E];
  load_slice<T, E>(pq, lead_q, a.V, slice, x);
  if (pp) load_slice<T, E>(pp, lead_q, a.V, slice, y);
  // (read by every workgroup, for the last one: behind its count they would be two more trips to memory)
  Child child{};
  if (t < 64) child = child_of<T>(a, b, i, v.kids);
  Part q, p{0.0, 0.0, -INFINITY, 0.f};
  if (first) {
    q = slice_sums64<T, E>(x, c, red, redm);
    __syncthreads();
    if (pp) p = slice_sums64<T, E>(y, c, red, redm);
  } else {
    const double A = v.Sq == 0.0 ? 0.0 : 1.0 / v.Sq, B = v.Sp == 0.0 ? 0.0 : v.a / v.Sp;
    if (distinct) {
      // the tried tokens are out of p's sum, and have no part in the other
      uint64_t left = v.kids;
      for (int j = v.state >> 8; j > 0; --j, left &= left - 1) {
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
    q.S = wave_sum(s[0] + s[1]);
    p.S = wave_sum(rest);
    if ((t & 63) == 0) {
      red[t >> 6] = q.S;
      red[4 + (t >> 6)] = p.S;
    }
    __syncthreads();
    q.S = red[0] + red[1] + (red[2] + red[3]);
    p.S = red[4] + red[5] + (red[6] + red[7]);
  }
  const int64_t at = ((int64_t)b * a.Q + i) * S;
  if (t == 0) {
    put(&w.sums[2 * (at + slice)], q.S);
    put(&w.sums[2 * (at + slice) + 1], p.S);
    if (first) {
      put(&w.maxima[2 * (at + slice)], q.m);
      put(&w.maxima[2 * (at + slice) + 1], p.m);
    }
    last_s = last_of(&w.arrived[(int64_t)b * (a.Q + 1) + i], (uint32_t)S);
  }
  __syncthreads();
  if (last_s) {
    if (t == 0) put(&w.arrived[(int64_t)b * (a.Q + 1) + i], 0u);
    // the first wavefront joins q's slices, the second p's
    const int h = t >> 6, lane = t & 63;
    if (h < 2) {
      // (a slice of -inf alone has no maximum, and one with NaN no sum)
      float m = -INFINITY;
      double sum = 0.0;
      for (int s = lane; s < S; s += 64) {
        const double g = get(&w.sums[2 * (at + s) + h]);
        if (!first) {
          sum += g;
          continue;
        }
        const float ms = get(&w.maxima[2 * (at + s) + h]), up = fmaxf(m, ms);
        if (m < up) sum = m == -INFINITY ? sum : sum * exp(((double)m - (double)up) * inv_t);
        if (!(ms == -INFINITY && g == 0.0)) sum += ms == up ? g : g * exp(((double)ms - (double)up) * inv_t);
        m = up;
      }
      if (first) {
        const float up = wave_max(m);
        if (m < up && m > -INFINITY) sum *= exp(((double)m - (double)up) * inv_t);
        m = up;
      }
      sum = wave_sum(sum);
      if (lane == 0) {
        joined[h] = sum;
        peaks[h] = m;
      }
    }
    __syncthreads();
    if (t < 64) {
      Node u = v;
      if (first) {
        u.Sq = joined[0];
        u.Sp = joined[1];
        u.mq = peaks[0] == -INFINITY ? 0.f : peaks[0];
        u.mp = peaks[1] == -INFINITY ? 0.f : peaks[1];
      } else {
        u.S = joined[0];
        // (weights below 2^-1000 are 0, for which the sum has 2^-1000)
        if (distinct) u.rest = v.Sp > 0.0 && joined[1] > 0x1p-960 ? joined[1] / v.Sp : 0.0;
      }
      tries(a, w, b, i, u, child, inv_t);
    }
  }
  __syncthreads();
}

// A step of every open node that the walk may come to and that lies at most `deep` steps below the root.  A node is out once another child of its parent is accepted or it is rejected.
// That may happen while this runs, and a workgroup that sees it leaves its slice out: then the node's
// count of slices never fills, and it stays open.  A workgroup's wavefronts have to agree on its nodes, as they meet in
// barriers at each: the first one reads the states, once, and hands the list to all.  (What else they read of a node on it
// stays as it is in this launch: it changes when the last of the node's slices is counted, and this workgroup's is one.)
template <class T, int E, int SUMS>
__global__ __launch_bounds__(kThreads) void tree_step_kernel(VerifyTreeArgs a, Tree w, int S, int R, int deep, Scale c, double inv_t) {
  __shared__ uint64_t list_s, kids_s[kNodes];
  const int slice = blockIdx.x % S, lane = threadIdx.x & 63;
  const int64_t id = blockIdx.x / S;
  const int b = (int)(id / R), worker = (int)(id % R);
  const Node* nodes = w.nodes + (int64_t)b * a.Q;
  if (threadIdx.x < 64) {
    const int state = lane < a.Q ? get(&nodes[lane].state) : kNone;
    const uint64_t kids_of = lane < a.Q ? nodes[lane].kids : 0;
    uint64_t open = kids_of;  // the children of node `lane` that are not out
    if (decided(state) != kOpen) open = decided(state) == kNone ? 0ull : 1ull << (decided(state) - 1);
    else
      for (int k = state >> 8; k > 0; --k) open &= open - 1;
    auto of = [](uint64_t v, int i) {
      return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, i) |
             (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), i) << 32;
    };
    const uint64_t inner = __ballot(open != 0);
    uint64_t alive = 1, todo = inner & 1;  // (a parent comes before its children)
    int depth = 0;
    while (todo) {
      const int i = __ffsll((unsigned long long)todo) - 1, below = __builtin_amdgcn_readlane(depth, i) + 1;
      const uint64_t more = below <= deep ? of(open, i) : 0;
      alive |= more;
      if (more >> lane & 1u) depth = below;
      todo = (todo & (todo - 1)) | (more & inner);
    }
    // (a node's workgroup is told by its place among all nodes with children, which does not change)
    const uint64_t kids = __ballot(kids_of != 0);
    const bool here = decided(state) == kOpen && kids_of != 0 && __popcll(kids & ((1ull << lane) - 1ull)) % R == worker;
    // (of the laws' own sums: nodes that have none yet)
    const uint64_t mine = __ballot(here && !(SUMS == kLaws && state >> 8)) & alive;
    kids_s[lane] = kids_of;
    if (lane == 0) list_s = mine;
  }
  __syncthreads();
  auto uniform = [](uint64_t v) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32)) << 32;
  };
  for (uint64_t mine = uniform(list_s); mine; mine &= mine - 1) {
    const int i = __ffsll((unsigned long long)mine) - 1;
    Node v{};
    if (SUMS == kLaws) {  // (nothing more is known of it yet)
      v.S = v.rest = 1.0;
      v.kids = uniform(kids_s[i]);
    } else {
      v = nodes[i];
      if (SUMS == kExcess && !v.steps) continue;
    }
    node_step<T, E, SUMS>(a, w, b, i, v, slice, S, c, inv_t);
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
    const int state = t < n ? decided(nodes[t].state) : kNone, next = state > kNone ? state - 1 : -1;
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
  // (a thread's first slice, mostly its only one, is read once)
  const double draw = draw_of(a, b), left0 = s0 < s1 ? get(&w.mass[2 * (base + s0)]) : 0.0,
               whole0 = s0 < s1 ? get(&w.mass[2 * (base + s0) + 1]) : 0.0;
  const float peak0 = s0 < s1 ? get(&w.peak[base + s0]) : 0.f;
  auto left_of = [&](int s) { return s == s0 ? left0 : get(&w.mass[2 * (base + s)]); };
  auto whole_of = [&](int s) { return s == s0 ? whole0 : get(&w.mass[2 * (base + s) + 1]); };
  auto peak_of = [&](int s) { return s == s0 ? peak0 : get(&w.peak[base + s]); };
  float m = -INFINITY;
  if (!inner) {
    for (int s = s0; s < s1; ++s)
      if (whole_of(s) != 0.0) m = fmaxf(m, peak_of(s));
    m = wave_max(m);
    if ((t & 63) == 0) redm[t >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(redm[0], redm[1]), fmaxf(redm[2], redm[3]));
  }
  auto factor = [&](int s) {
    if (inner) return 1.0;
    const double z = ((double)peak_of(s) - (double)m) * inv_t;
    return z < -700.0 ? 0.0 : exp(z);
  };
  bool use_q = false;
  auto mass_of = [&](int s) {
    const double g = use_q ? whole_of(s) : left_of(s);
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
  const double goal = draw * all;
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

// Workgroups share a tree's nodes with children: half as many as nodes take all of them, in two turns where the
// tree is a chain, and four the ones that a walk may still come to.
inline int many(int Q) { return Q > 1 ? Q / 2 : 1; }
inline int few(int Q) { return Q > 4 ? 4 : Q > 1 ? Q - 1 : 1; }
// Whether the root's law comes first, then its children's that are left, then the rest's: two launches more, and
// most nodes out before they are summed.  A chain's next node is never out before the last one is summed: there the
// stages go to depths 1, 3, 7 and so on.  In us (graphs), at once / in stages, trees x nodes x vocabulary:
//   1 x 12 x 32000 36 / 51     4 x 32 x 131072 49 / 60    16 x 12 x 131072 90 / 89   32 x 32 x 32000 98 / 96
//   8 x 32 x 131072 89 / 92    64 x 16 x 50001 132 / 132  32 x 12 x 131072 129 / 120 16 x 32 x 131072 124 / 115
//   32 x 32 x 131072 190 / 139
//   given: 24 x 24 x 50001 44 / 51   8 x 32 x 131072 45 / 48   16 x 24 x 131072 56 / 58   64 x 24 x 50001 80 / 70
//   64 x 64 x 131072 386 / 115
//   chains: 20 x 18 x 60620 81 / 91   4 x 64 x 131072 114 / 61   32 x 32 x 52733 130 / 138   25 x 26 x 147437 183 / 145 (an
//   earlier form with children of the root and the rest alone: 174)
inline bool in_stages(const VerifyTreeArgs& a) {
  return (int64_t)a.B * a.Q * a.V >= (a.max_children == 1 ? 24ll << 20 : 40ll << 20);
}

struct TreeWs {
  size_t nodes, arrived, chance, sums, maxima, mass, peak, bytes;
};
TreeWs tree_layout(int B, int Q, int V) {
  const size_t S = (size_t)slices(V, per_thread(B, V)), n = (size_t)B * Q;  // (the most: more rows have no smaller slices)
  TreeWs w;
  w.nodes = 0;
  w.arrived = w.nodes + up256(sizeof(Node) * n);
  w.chance = w.arrived + up256(sizeof(uint32_t) * (n + B));
  w.sums = w.chance + up256(sizeof(float) * n);
  w.maxima = w.sums + up256(2 * sizeof(double) * n * S);
  w.mass = w.maxima + up256(2 * sizeof(float) * n * S);
  w.peak = w.mass + up256(2 * sizeof(double) * (size_t)B * S);
  w.bytes = w.peak + up256(sizeof(float) * (size_t)B * S);
  return w;
}

// A step, by `workers` slices' workgroups a tree.
template <class T, int E, int SUMS>
hipError_t step_run(const char* name, const VerifyTreeArgs& a, const Tree& w, int deep, int workers, double inv_t, hipStream_t s) {
  const int S = slices(a.V, E);
  return launch_timed(name, tree_step_kernel<T, E, SUMS>, dim3((unsigned)((int64_t)a.B * workers * S)), dim3(kThreads), s, a, w, S,
                      workers, deep, scale_of(inv_t), inv_t);
}
template <class T, int SUMS>
hipError_t step_of(const char* name, const VerifyTreeArgs& a, const Tree& w, int deep, int workers, double inv_t, hipStream_t s) {
  return per_thread((int64_t)a.B * workers, a.V) == 32 ? step_run<T, 32, SUMS>(name, a, w, deep, workers, inv_t, s)
                                                       : step_run<T, 8, SUMS>(name, a, w, deep, workers, inv_t, s);
}
template <class T>
hipError_t laws_run(const VerifyTreeArgs& a, const Tree& w, double inv_t, hipStream_t s) {
  const bool given = a.draws == SD_TREE_GIVEN;  // (no sum behind the laws')
  hipError_t e;
  if (in_stages(a)) {
    const bool chain = a.max_children == 1;
    auto stage = [&](const char* name, int deep) {
      if (e == hipSuccess)
        e = given || chain ? step_of<T, kLaws>(name, a, w, deep, few(a.Q), inv_t, s)
                           : step_of<T, kBoth>(name, a, w, deep, few(a.Q), inv_t, s);
    };
    e = step_of<T, kLaws>("tree_root", a, w, 0, 1, inv_t, s);
    for (int deep = 1; deep < (chain ? a.Q - 2 : 2); deep = 2 * deep + 1) stage("tree_near", deep);
    stage("tree_rest", a.Q);
  } else {
    e = step_of<T, kLaws>("tree_laws", a, w, a.Q, many(a.Q), inv_t, s);
  }
  if (given) return e;
  for (int k = 1; k < a.max_children && k < a.Q - 1 && e == hipSuccess; ++k)
    e = step_of<T, kExcess>("tree_round", a, w, a.Q, few(a.Q), inv_t, s);
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
  return (int64_t)B * (many(Q) > few(Q) ? many(Q) : few(Q)) * slices(V, per_thread(B, V));
}

hipError_t verify_tree_launch(const VerifyTreeArgs& a, sd_type type, double temperature, void* ws, hipStream_t s) {
  const double inv_t = 1.0 / temperature;
  const TreeWs l = tree_layout(a.B, a.Q, a.V);
  char* base = static_cast<char*>(ws);
  const Tree w{reinterpret_cast<Node*>(base + l.nodes),   reinterpret_cast<uint32_t*>(base + l.arrived),
               reinterpret_cast<float*>(base + l.chance), reinterpret_cast<double*>(base + l.sums),
               reinterpret_cast<float*>(base + l.maxima), reinterpret_cast<double*>(base + l.mass),
               reinterpret_cast<float*>(base + l.peak)};
  hipError_t e = launch_timed("tree_plan", tree_plan_kernel, dim3((unsigned)a.B), dim3(64), s, a, w);
  if (e != hipSuccess) return e;
  return by_type(type, [&](auto tag) {
    typedef decltype(tag) T;
    const hipError_t e = a.Q > 1 ? laws_run<T>(a, w, inv_t, s) : hipSuccess;
    if (e != hipSuccess) return e;
    return per_thread(a.B, a.V) == 32 ? draw_run<T, 32>(a, w, inv_t, s) : draw_run<T, 8>(a, w, inv_t, s);
  });
}

}  // namespace sd
