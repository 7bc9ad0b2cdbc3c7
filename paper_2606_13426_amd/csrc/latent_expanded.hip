// Causal attention of ragged sequences with per-head keys and values and one
// rotary key a token that all heads share (the expanded form of latent
// attention), for prompts (gfx950).
//
// A workgroup of four wavefronts takes 128 query rows of one head of one
// sequence, a wavefront 32 of them, and walks the keys 64 at a time:
//   S^T [keys][rows] = K Q^T      on v_mfma_f32_32x32x16, Q in registers
//   P = 2^{S c - m}, c = scale log2(e)
//   O^T [values][rows] += V^T P^T
// In both results a lane holds one row (of the two halves of a wavefront, the same
// row twice with other keys), so the softmax takes one exchange between the
// halves, and S^T's registers are P^T's operand as they are: the instruction's
// places along k are free to mean any keys as long as V^T, read by transposing LDS
// loads, has the same order.  No value of S or P passes through LDS.
//
// m is a reference and not the maximum: it moves when a score exceeds it by more than
// it is allowed to (reach), so the rescaling of O is left out of almost every tile.
// P is rounded to the operands' type, half a step a weight (the instruction takes both
// operands of one type); the weights' sum is of the float32 ones.
//
// Tiles (K rotary and not, V) come by loads that write LDS directly, into the other
// of two buffers while this one is multiplied; one barrier a tile.  80 KB of LDS
// and at most 256 registers: two workgroups a compute unit, so one's products
// cover the other's softmax.
//
// Where the rows' tiles do not fill the compute units the keys are split too, and
// expanded_join_kernel joins the parts.
//
// What bounds it, on MI355X: matrix and vector instructions together (the matrix cores
// are busy for 55 % of the time, vector instructions issue for 47 %), at clocks that
// such a load pulls down.  2 prompts of 6144 tokens, 32 heads, bf16: 430 to 530 us from a cool
// to a warm card, 0.80 to 0.99 PFLOP/s; 1000 rows on 8500 keys, 16 heads: 90 us and 8 for
// the join, 0.87 PFLOP/s.  Short prompts are their loads' latency: 33 of up to 211
// tokens, 35 us, 2.4 TB/s.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.hpp"
#include "latent_common.hpp"

namespace sd {
namespace {

using namespace latent;

constexpr int kRows = 128;

struct Expanded {
  int n, H, dn, dr, dv, Tq, Tk;
  float c;     // |scale| log2(e)
  uint32_t flip;  // sign bits of a pair, to negate q where scale is negative
  const uint16_t *q, *k, *kr, *v;
  int64_t qt, qh, kt, kh, krt, vt, vh;
  const int32_t *cu_q, *cu_k;
  uint16_t* out;
  int64_t ot, oh;
  float* lse;
  int tiles, split;
  float* part;   // [split][Tq][H][DV] unnormalised O
  float2* stat;  // [split][Tq][H] (reference, sum)
};

__device__ __forceinline__ int offset_of(const int32_t* cu, int i, int total) { return min(max(load_global<int32_t>(cu + i), 0), total); }

template <class T, int DN, int DV>
__global__ __launch_bounds__(kThreads, 2) void expanded_kernel(Expanded a) {
  constexpr int DK = DN + kRope, KS = DK / 16, NV = DV / 32;
  constexpr int CN = DN / 8, CR = kRope / 8, CV = DV / 8;  // 16-byte pieces a token in the three parts
  constexpr int kKr = kTile * DN * 2, kV = kKr + kTile * kRope * 2, kStage = kV + kTile * DV * 2;
  __shared__ __align__(16) char buf[2 * kStage];
  const int t = threadIdx.x, w = (int)uniform((uint32_t)t >> 6), lane = t & 63, n = lane & 31, h = lane >> 5;

  // the tiles of a head from the last to the first, a head's tiles on one XCD
  const int id = xcd_tile((int)(gridDim.x * gridDim.y * gridDim.z));
  const int part = id % a.split, tile = a.tiles - 1 - id / a.split % a.tiles, head = id / a.split / a.tiles;
  // Sequence b's tiles are numbered from cu_q[b] / 128 + b, which rises: the sequences that begin at or before
  // this one's are counted by the last of 64 parts of those in question at a time.  (Every workgroup over
  // all sequences: 26.5 ms for 16384 of 64 rows, 16 heads.)
  int before = 0;
  for (int left = a.n, step; left > 0; left = step > 1 ? min(step, left) : 0) {
    step = (left + 63) / 64;
    const int at = before + (lane + 1) * step - 1;
    const bool here = (lane + 1) * step <= left;
    const int parts = __popcll(__ballot(here && offset_of(a.cu_q, here ? at : 0, a.Tq) / kRows + at <= tile));
    before += parts * step;
    left -= parts * step;
  }
  const int b = __builtin_amdgcn_readfirstlane(max(before - 1, 0));
  const int qb = offset_of(a.cu_q, b, a.Tq), kb = offset_of(a.cu_k, b, a.Tk);
  const int nq = max(offset_of(a.cu_q, b + 1, a.Tq) - qb, 0), nk = max(offset_of(a.cu_k, b + 1, a.Tk) - kb, 0);
  const int q0 = (tile - (qb / kRows + b)) * kRows;
  if (q0 < 0 || q0 >= nq) return;
  const int shift = nk - nq + 1;  // row i sees keys below i + shift
  const int end = min(max(min(q0 + kRows, nq) - 1 + shift, 0), nk);
  const int all = (end + kTile - 1) / kTile;
  const int t0 = (int)((int64_t)all * part / a.split), t1 = (int)((int64_t)all * (part + 1) / a.split);

  const int row = q0 + 32 * w + n;
  const bool real = row < nq;
  const int lim = real ? min(max(row + shift, 0), nk) : 0;
  // the least limit of the workgroup's rows; tiles that reach past it have keys that not all its rows see
  const int g_lo = min(max(q0 + shift, 0), nk);
  auto mixed = [&](int tl) { return (tl + 1) * kTile > g_lo; };
  const int w_lo = min(max(q0 + 32 * w + shift, 0), nk);  // the least limit of this wavefront's rows
  const bool idle = q0 + 32 * w >= nq;

  u32x4 qf[KS];
  {
    const uint16_t* src = a.q + (int64_t)(qb + min(row, nq - 1)) * a.qt + (int64_t)head * a.qh;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int col = 16 * k + 8 * h;
      const int at = col < DN ? (col < a.dn ? col : -1) : (col - DN < a.dr ? a.dn + col - DN : -1);
      // (loads are not branched around, so that all are in flight together)
      qf[k] = load_global<u32x4>(src + (at >= 0 ? at : 0));
      qf[k] = at >= 0 ? qf[k] : u32x4{0u, 0u, 0u, 0u};
      qf[k] ^= a.flip;
    }
  }
  f32x16 o[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) o[k] = f32x16{};
  float m = -INFINITY, l = 0.f;

  // Piece 64 (w + 4 i) + lane of each part of a tile: its token, and the column (permuted among eight).
  const Global gk = (Global)(a.k + (int64_t)kb * a.kt + (int64_t)head * a.kh);
  const Global gr = (Global)(a.kr + (int64_t)kb * a.krt);
  const Global gv = (Global)(a.v + (int64_t)kb * a.vt + (int64_t)head * a.vh);
  const Lds lds = lds_of(buf);
  const bool padded = a.dn != DN || a.dr != kRope || a.dv != DV;
  uint32_t off_n[CN / 4], off_r[CR / 4], off_v[CV / 4];
  auto rare = [&](int v) {  // (what the loop's rare paths compute from it is not kept in registers)
    asm volatile("" : "+v"(v));
    return v;
  };
  auto place = [&](int P, int i, int* tok) {
    const int s = 64 * (w + 4 * i) + lane, pc = s % P;
    *tok = s / P;
    return ((pc & ~7) | ((pc ^ perm(*tok)) & 7)) * 8;
  };
  auto set_offsets = [&](int P, int64_t stride, int d, uint32_t* to) {
    for (int i = 0; i < P / 4; ++i) {
      int tok;
      const int col = place(P, i, &tok);
      // (a column that is not there lies past every view's end: nothing is read for it)
      to[i] = col < d ? 2u * (uint32_t)(tok * (int)stride + col) : 0x80000000u;
    }
  };
  set_offsets(CN, a.kt, a.dn, off_n);
  set_offsets(CR, a.krt, a.dr, off_r);
  set_offsets(CV, a.vt, a.dv, off_v);
  // piece i of a wavefront goes to 1024 (w + 4 i): four wavefronts side by side
  // The three views of a tile, for loads that go out one after another (next_load); `on` is 0 where
  // the tile is of another kind (its keys end in it) and loaded here.
  struct Load {
    u32x4 n, r, v;
    uint32_t dst;
    uint64_t on;
  };
  auto base_of = [&](Global base, int64_t stride, int tl) { return base + (int64_t)tl * kTile * stride * 2; };
  auto slow_part = [&](int P, Global base, int64_t stride, int d, int tl, Lds dst) {
    const Global src = base_of(base, stride, tl);
    const int last = nk - 1 - tl * kTile, ln = rare(lane);  // places behind the last key repeat it; their weights are 0
#pragma unroll 1
    for (int i = 0; i < P / 4; ++i) {
      const int s = 64 * (w + 4 * i) + ln, pc = s % P, tok = s / P, col = ((pc & ~7) | ((pc ^ perm(tok)) & 7)) * 8;
      if (col < d) load_lds(src + 2u * (uint32_t)(min(tok, last) * (int)stride + col), dst + 1024 * (w + 4 * i));
    }
  };
  auto start_load = [&](int tl, Lds dst, bool want) -> Load {
    Load ld;
    const bool fast = tl * kTile + kTile <= nk;
    if (want && !fast) {
      slow_part(CN, gk, a.kt, a.dn, tl, dst);
      slow_part(CR, gr, a.krt, a.dr, tl, dst + kKr);
      slow_part(CV, gv, a.vt, a.dv, tl, dst + kV);
    }
    ld.n = lds_view((const void*)base_of(gk, a.kt, tl), 2 * ((kTile - 1) * a.kt + a.dn));
    ld.r = lds_view((const void*)base_of(gr, a.krt, tl), 2 * ((kTile - 1) * a.krt + a.dr));
    ld.v = lds_view((const void*)base_of(gv, a.vt, tl), 2 * ((kTile - 1) * a.vt + a.dv));
    ld.dst = lds_address(dst + 1024 * w);
    ld.on = (uint64_t)0 - (uint64_t)uniform(fast && want ? 1u : 0u);
    return ld;
  };
  constexpr int kLoads = (CN + CR + CV) / 4;
  auto next_load = [&](const Load& ld, auto i) {
    constexpr int I = decltype(i)::value;
    if constexpr (I < CN / 4)
      load_lds_view<4096 * I>(ld.n, off_n[I], ld.dst, ld.on);
    else if constexpr (I < (CN + CR) / 4)
      load_lds_view<4096 * (I - CN / 4) + kKr>(ld.r, off_r[I - CN / 4], ld.dst, ld.on);
    else
      load_lds_view<4096 * (I - (CN + CR) / 4) + kV>(ld.v, off_v[I - (CN + CR) / 4], ld.dst, ld.on);
  };
  if (padded) {
    // pieces that no load writes are zero in both buffers
    for (int i = t; i < 2 * kStage / 16; i += kThreads) reinterpret_cast<u32x4*>(buf)[i] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
  }
  if (t0 < t1) {
    const Load ld = start_load(t0, lds, true);
    each<kLoads>([&](auto i) { next_load(ld, i); });
  }

  // what a lane reads of a tile, in bytes: of key n (and n + 32) piece 2 k + h; of values four tokens by
  // sixteen columns, of which the lanes from 16 and 48 on take the upper sixteen of a block of 32
  const int kx = h ^ perm(n), krow = n * DN * 2 + kx * 16, rrow = kKr + n * kRope * 2 + kx * 16;
  const int vtok = 4 * h + ((lane & 15) >> 2), vch = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
  const int vrow[2] = {vtok * DV * 2 + (vch ^ perm(vtok)) * 16 + 8 * (lane & 1),
                       vtok * DV * 2 + ((vch + 4) ^ perm(vtok)) * 16 + 8 * (lane & 1)};

  for (int tl = t0; tl < t1; ++tl) {
    const Lds here = lds + (tl - t0 & 1) * kStage;
    __builtin_amdgcn_s_waitcnt(0);
    lds_barrier();
    Load ld = start_load(min(tl + 1, t1 - 1), lds + (tl - t0 + 1 & 1) * kStage, tl + 1 < t1);
    if (idle && !mixed(tl)) {
      // a wavefront without rows only loads; in mixed tiles it takes part in the look for infinities below
      // (where rows see nothing of a tile that others see, it is mixed)
      each<kLoads>([&](auto i) { next_load(ld, i); });
      continue;
    }

    f32x16 s[2] = {f32x16{}, f32x16{}};
    {
      // a step's pieces are read while the two before it are multiplied; the next tile's loads go out between
      __builtin_amdgcn_s_setprio(1);
      u32x4 kf[3][2];
      auto read = [&](int k) {
        const bool own = k < DN / 16;
        const int kk = own ? k : k - DN / 16;
#pragma unroll
        for (int b2 = 0; b2 < 2; ++b2)
          kf[k % 3][b2] = lds_read<u32x4>(here + (own ? krow : rrow) + (own ? 32 * b2 * DN * 2 : 32 * b2 * kRope * 2) +
                                          (kk >> 2) * 128 + (((2 * (kk & 3)) ^ kx) - kx) * 16);
      };
      read(0);
      read(1);
      each<KS>([&](auto step) {
        constexpr int k = decltype(step)::value;
        if (k + 2 < KS) read(k + 2);
        __builtin_amdgcn_sched_barrier(0);
        each<kLoads>([&](auto i) {
          if constexpr (i * KS / kLoads == k) next_load(ld, i);
        });
#pragma unroll
        for (int b2 = 0; b2 < 2; ++b2) s[b2] = T::mfma32(kf[k % 3][b2], qf[k], s[b2]);
        __builtin_amdgcn_sched_barrier(0);
      });
    }
#pragma unroll
    for (int b2 = 0; b2 < 2; ++b2) asm volatile("" : "+v"(s[b2]));  // taken up before any branch
    __builtin_amdgcn_s_setprio(0);
    const bool edge = (tl + 1) * kTile > w_lo;
    if (edge) {
#pragma unroll
      for (int b2 = 0; b2 < 2; ++b2)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[b2][i] = tl * kTile + 32 * b2 + 8 * (i >> 2) + 4 * h + (i & 3) < lim ? s[b2][i] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[1][i]);
    mx = across(mx, true, true) * a.c;
    // (a NaN score passes the maximum over and makes its row NaN by its weight)
    const bool up = mx > reach<T>(m);
    if (__any(up)) {
      const float to = up ? reference<T>(mx) : m, f = up ? __builtin_amdgcn_exp2f(m - to) : 1.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) o[k] *= f;
      l *= f;
      m = to;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    u32x4 pf[4];
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    auto weigh = [&](int b2, int i) {  // scores i and i + 1 of a half
      const float p0 = __builtin_amdgcn_exp2f(__fmaf_rn(s[b2][i], a.c, -ref));
      const float p1 = __builtin_amdgcn_exp2f(__fmaf_rn(s[b2][i + 1], a.c, -ref));
      sum[i & 2] += p0;
      sum[(i & 2) + 1] += p1;
      pf[2 * b2 + (i >> 3)][(i & 7) >> 1] = T::pack(p0, p1);
    };
#pragma unroll
    for (int i = 0; i < 16; i += 2) weigh(0, i);

    // A key that some rows of the workgroup see and others do not: its weight for those is 0, and 0
    // times an infinity or NaN in its value is not.  All wavefronts look and find the same.
    if (mixed(tl)) {
      const int from = max(g_lo - tl * kTile, 0), ln = rare(lane);
      uint32_t bad = 0;
      for (int i = ln; i < (kTile - from) * CV; i += 64) {
        const u32x4 v = lds_read<u32x4>(here + kV + from * DV * 2 + 16 * i);
        bad |= (lawless<T>(v[0]) | lawless<T>(v[1])) | (lawless<T>(v[2]) | lawless<T>(v[3]));
      }
      if (__any((bad & 0x80008000u) != 0)) {
        // what they give to the rows that see them, and zeros in their place
        const int hh = ln >> 5, row_lim = lim - tl * kTile;
#pragma clang loop unroll(disable)
        for (int j = from; j < kTile; ++j) {
          // the row's weight for key j, as the product takes it: its score is one of this lane's or of the
          // row's other lane's
          const int at = 16 * (j >> 5) + 4 * (j >> 3 & 3) + (j & 3);
          float score = 0.f;
#pragma unroll
          for (int i = 0; i < 32; ++i) score = i == at ? s[i >> 4][i & 15] : score;
          uint32_t lower = __builtin_bit_cast(uint32_t, score), upper = lower;
          swap32(lower, upper);
          score = __builtin_bit_cast(float, j >> 2 & 1 ? upper : lower);
          const float p = T::value((uint16_t)T::pack(__builtin_amdgcn_exp2f(__fmaf_rn(score, a.c, -ref)), 0.f));
#pragma unroll
          for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int col = 32 * k + 8 * (i >> 2) + 4 * hh + (i & 3), pc = (col >> 3 & ~7) | ((col >> 3 ^ perm(j)) & 7);
              const uint32_t v = lds_read<uint16_t>(here + kV + j * DV * 2 + pc * 16 + 2 * (col & 7));
              if ((v & T::kExponent) == T::kExponent && j < row_lim) o[k][i] += p * T::value((uint16_t)v);
            }
        }
        lds_barrier();
        for (int i = from * DV + rare(t); i < kTile * DV; i += kThreads) {
          const Lds at = here + kV + 2 * i;
          if ((lds_read<uint16_t>(at) & T::kExponent) == T::kExponent) *(__attribute__((address_space(3))) uint16_t*)at = 0;
        }
        lds_barrier();
      }
    }
    {
      // Two blocks' values are read while one is multiplied, and the second half's weights are made in
      // the first half's products' time.  The products go first where both wavefronts of a SIMD have
      // something to issue.
      __builtin_amdgcn_s_setprio(1);
      u32x4 vf[3];
      auto read = [&](int i) {
        const Lds src = here + kV + (i / NV) * 16 * DV * 2 + vrow[i % NV & 1] + (i % NV >> 1) * 128;
        const u32x2 lo = lds_read_tr(src), hi = lds_read_tr(src + 8 * DV * 2);
        vf[i % 3] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      };
      read(0);
      read(1);
#pragma unroll
      for (int i = 0; i < 4 * NV; ++i) {
        if (i + 2 < 4 * NV) read(i + 2);
        __builtin_amdgcn_sched_barrier(0);
        o[i % NV] = T::mfma32(vf[i % 3], pf[i / NV], o[i % NV]);
        if (i < 2 * NV) {
#pragma unroll
          for (int j = 0; j < 4 / NV; ++j) weigh(1, 2 * (i * (4 / NV) + j));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    // wait states for a read of the last results behind the loop's branch
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15");
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  }

  l = across(l, true, false);
  if (!real) return;
  const int64_t at = (int64_t)(qb + row) * a.H + head;
  if (a.split > 1) {
    float* dst = a.part + ((int64_t)part * a.Tq * a.H + at) * DV;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(dst + 32 * k + 2 * i + 4 * h) = f32x4{o[k][i], o[k][i + 1], o[k][i + 2], o[k][i + 3]};
    if (h == 0) a.stat[(int64_t)part * a.Tq * a.H + at] = make_float2(m, l);
    return;
  }
  const float f = l > 0.f ? 1.f / l : l != l ? NAN : 0.f;
  uint16_t* dst = a.out + (int64_t)(qb + row) * a.ot + (int64_t)head * a.oh;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int col = 32 * k + 2 * i + 4 * h;
      if (col < a.dv)
        *reinterpret_cast<u32x2*>(dst + col) = u32x2{T::pack(o[k][i] * f, o[k][i + 1] * f), T::pack(o[k][i + 2] * f, o[k][i + 3] * f)};
    }
  if (a.lse && h == 0) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The parts of rows whose keys were split, joined: DV / 4 threads a row.
template <class T, int DV>
__global__ __launch_bounds__(kThreads) void expanded_join_kernel(Expanded a) {
  constexpr int kWays = DV / 4;
  const int64_t at = (int64_t)blockIdx.x * (kThreads / kWays) + threadIdx.x / kWays, rows = (int64_t)a.Tq * a.H;
  if (at >= rows) return;
  const int tok = (int)(at / a.H), head = (int)(at % a.H), c = threadIdx.x % kWays * 4;
  // rows before the first sequence and behind the last are nobody's
  if (tok < offset_of(a.cu_q, 0, a.Tq) || tok >= offset_of(a.cu_q, a.n, a.Tq)) return;
  float m = -INFINITY;
  for (int s = 0; s < a.split; ++s) m = fmaxf(m, a.stat[s * rows + at].x);
  const float ref = m == -INFINITY ? 0.f : m;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int s = 0; s < a.split; ++s) {
    const float2 st = a.stat[s * rows + at];
    const float f = __builtin_amdgcn_exp2f(st.x - ref);
    l += st.y * f;
    o += *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * DV + c) * f;
  }
  const float f = l > 0.f ? 1.f / l : l != l ? NAN : 0.f;
  if (c < a.dv)
    *reinterpret_cast<u32x2*>(a.out + (int64_t)tok * a.ot + (int64_t)head * a.oh + c) =
        u32x2{T::pack(o[0] * f, o[1] * f), T::pack(o[2] * f, o[3] * f)};
  if (a.lse && c == 0) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int tiles_of(int Tq, int n) { return Tq / kRows + n; }
// The parts that a row's keys are split into: as many as fill 256 compute units
// with two workgroups, at most 8, and none of fewer than 256 keys where all have
// the same number.  In us: 1000 rows on 8000 keys, 16 heads: 185 whole, 93 in 4 parts,
// 107 in 8; 32 heads: 212 whole, 172 in 2, 193 in 4; 4 x 512 rows on 2512 keys, 16
// heads: 86 whole, 69 in 2.
inline int split_of(int n, int H, int Tq, int Tk) {
  const int64_t groups = ((int64_t)Tq + kRows - 1) / kRows * H;
  int s = 1;
  while (s < 8 && groups * 2 * s <= 512 && Tk / n >= 512 * s) s *= 2;
  return s;
}
inline int padded_dv(int dn, int dv) { return dn <= 64 && dv <= 64 ? 64 : 128; }

template <class T>
hipError_t run(const Expanded& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.tiles * a.split), (unsigned)a.H), block(kThreads);
  const bool small = padded_dv(a.dn, a.dv) == 64;
  hipError_t e = small ? launch_timed("latent_expanded", expanded_kernel<T, 64, 64>, grid, block, s, a)
                       : launch_timed("latent_expanded", expanded_kernel<T, 128, 128>, grid, block, s, a);
  if (e != hipSuccess || a.split == 1) return e;
  const int per = kThreads / (small ? 16 : 32);
  const dim3 jgrid((unsigned)(((int64_t)a.Tq * a.H + per - 1) / per));
  return small ? launch_timed("latent_expanded_join", expanded_join_kernel<T, 64>, jgrid, block, s, a)
               : launch_timed("latent_expanded_join", expanded_join_kernel<T, 128>, jgrid, block, s, a);
}

}  // namespace

size_t expanded_ws_bytes(int n, int H, int dn, int dv, int Tq, int Tk) {
  const int split = split_of(n, H, Tq, Tk);
  if (split == 1) return 0;
  const size_t rows = (size_t)split * Tq * H;
  return up256(rows * padded_dv(dn, dv) * sizeof(float)) + up256(rows * sizeof(float2));
}
// Workgroups a head.
int64_t expanded_groups(int n, int H, int Tq, int Tk) {
  return (int64_t)tiles_of(Tq, n) * split_of(n, H, Tq, Tk);
}

hipError_t expanded_launch(int n, int H, int dn, int dr, int dv, sd_type type, double scale, int Tq, const void* q,
                           sd_stride_h qs, int Tk, const void* k, sd_stride_h ks, const void* kr, int64_t kr_stride,
                           const void* v, sd_stride_h vs, const int32_t* cu_q, const int32_t* cu_k, void* out,
                           sd_stride_h os, float* lse, void* ws, hipStream_t s) {
  Expanded a;
  a.n = n;
  a.H = H;
  a.dn = dn;
  a.dr = dr;
  a.dv = dv;
  a.Tq = Tq;
  a.Tk = Tk;
  // |scale| at least 1e-30, so that a masked score stays -inf where scale is 0
  a.c = (float)fmax(fabs(scale) * 1.44269504088896340736, 1e-30);
  a.flip = scale < 0.0 ? 0x80008000u : 0u;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.kr = static_cast<const uint16_t*>(kr);
  a.v = static_cast<const uint16_t*>(v);
  a.qt = qs.row;
  a.qh = qs.head;
  a.kt = ks.row;
  a.kh = ks.head;
  a.krt = kr_stride;
  a.vt = vs.row;
  a.vh = vs.head;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.out = static_cast<uint16_t*>(out);
  a.ot = os.row;
  a.oh = os.head;
  a.lse = lse;
  a.tiles = tiles_of(Tq, n);
  a.split = split_of(n, H, Tq, Tk);
  a.part = static_cast<float*>(ws);
  a.stat = reinterpret_cast<float2*>(static_cast<char*>(ws) +
                                     up256((size_t)a.split * Tq * H * padded_dv(dn, dv) * sizeof(float)));
  return type == SD_TYPE_BF16 ? run<Bf16>(a, s) : run<F16>(a, s);
}

}  // namespace sd
