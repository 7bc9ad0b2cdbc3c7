// Attention of a few query rows a sequence over a cache of one shared latent
// vector a token (gfx950): keys are the whole vector (latent and rotary part),
// values its latent part.
//
// A workgroup of four wavefronts takes 16 R rows (row, head pairs) of one
// sequence and a run of its tokens, 64 at a time.  A tile of the cache enters LDS
// once and serves both products, so a token's bytes come from HBM once for all
// the rows of a workgroup:
//   S^T [tokens][rows] = C Q^T   wavefront w: tokens 16 w .. 16 w + 15, all rows;
//                                its part of Q stays in registers
//   P = e^{S - m}                running maxima over the four wavefronts by LDS
//   O^T [latent][rows] = C^T P^T wavefront w: a quarter of the latent columns,
//                                all rows, accumulators in registers
// on v_mfma_f32_16x16x32.  In both results a lane holds one row of each block of
// 16, so its maximum, sum and rescaling need no exchange inside the products.
// C^T is read by transposing LDS loads; the order in which the 32 tokens of a
// step meet the instruction's k places is the one those loads give, and P is
// stored to match.
//
// Tiles come by loads that write LDS directly, the next one while this one is
// multiplied.  A token's 16-byte pieces are permuted inside each 128 bytes by
// perm(token), which the lanes' global addresses do, so that both products'
// reads meet every bank once.
//
// The tokens of all sequences form one list that is cut into equal runs, one a
// workgroup (a team of workgroups where one sequence's rows take several: they
// run on one XCD, whose L2 then holds the tile for all of them).  A run may end
// inside a sequence: its part is left in the workspace and joined by
// latent_join_kernel.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "latent_common.hpp"

namespace sd {
namespace latent {

constexpr int kGroups = 256;  // workgroups: one a compute unit (the tiles fill its LDS)

// How the rows of a sequence are dealt to workgroups: blocks of 16 R rows, teams
// of `team` blocks that walk the same tokens, `supers` teams' worth a sequence.
struct Plan {
  int R, blocks, team, supers, teams;
};
inline Plan plan(int Q, int H) {
  const int64_t rows = (int64_t)Q * H;
  Plan p;
  p.R = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.blocks = (int)((rows + 16 * p.R - 1) / (16 * p.R));
  p.team = p.blocks % 4 == 0 ? 4 : p.blocks % 2 == 0 ? 2 : p.blocks == 3 ? 3 : 1;
  p.supers = p.blocks / p.team;
  p.teams = 8 * (kGroups / 8 / p.team);
  return p;
}

struct Args {
  int B, Q, H, dc, dr;
  float c;  // scale log2(e)
  const uint16_t* q;
  int64_t qs, qr, qh;
  const uint16_t* cache;
  int64_t page_stride, token_stride;
  int n_pages, page_size;
  const int32_t* pages;  // null: page b is sequence b
  int64_t pages_stride;
  int capacity;  // tokens that a sequence's pages hold
  const int32_t* lens;
  const int32_t* rows;  // null: Q
  uint16_t* out;
  int64_t os, orow, oh;
  float* lse;  // null, or [B][Q][H]
  Plan p;
  float* part;     // [kGroups][2][16 R][DC] unnormalised O
  float2* stat;    // [kGroups][2][16 R] (maximum in log2 units, sum)
  int32_t* first;  // [B][supers] 2 team + slot of the run that starts the sequence; -1: one run did it all
  int32_t* last;   // [B][supers] the team that ends it
  int64_t* total;  // the list's tiles
};

__device__ __forceinline__ int length_of(const Args& a, int b) { return min(max(a.lens[b], 0), a.capacity); }
__device__ __forceinline__ int rows_of(const Args& a, int b) {
  return a.rows ? min(max(a.rows[b], 0), a.Q) : a.Q;
}
// The first tile of a team's run of a list of `total`.
__device__ __forceinline__ int64_t run_begin(int64_t total, int team, int teams) { return total * team / teams; }
__device__ __forceinline__ int tiles_of(int len) { return (len + kTile - 1) / kTile; }

template <class T, int R, int DC>
__global__ __launch_bounds__(kThreads, 1) void latent_kernel(Args a) {
  constexpr int C = (DC + kRope) / 8;      // 16-byte pieces of a token
  constexpr int KS = (DC + kRope) / 32;    // steps of 32 columns of Q
  constexpr int NB = DC / 64;              // blocks of 16 latent columns of a wavefront
  constexpr int NL = C / 4;                // loads of 64 pieces for a wavefront's 16 tokens
  static_assert(C % 8 == 0 && DC % 128 == 0, "whole 128-byte segments, and whole blocks a wavefront");
  __shared__ __align__(16) uint16_t tile[2][kTile * C * 8];
  __shared__ __align__(16) uint16_t pl[16 * R * kTile];
  __shared__ float red[4][16 * R];
  __shared__ int64_t scan[4];
  __shared__ int64_t found[2];

  const int t = threadIdx.x, w = t >> 6, lane = t & 63, n = lane & 15, g = lane >> 4;
  const int L = blockIdx.x, per = kGroups / 8 / a.p.team;
  const int i8 = L / 8, team = (L % 8) * per + i8 / a.p.team, member = i8 % a.p.team;
  if (i8 >= per * a.p.team) return;

  // this team's run of the list of all sequences' tiles
  int64_t mine = 0;
  const int bper = (a.B + kThreads - 1) / kThreads, b0 = min(t * bper, a.B), b1 = min(b0 + bper, a.B);
  for (int b = b0; b < b1; ++b) mine += (int64_t)tiles_of(length_of(a, b)) * a.p.supers;
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up((long long)upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) scan[w] = upto;
  __syncthreads();
  for (int i = 0; i < w; ++i) upto += scan[i];
  const int64_t total = scan[0] + scan[1] + scan[2] + scan[3];
  const int64_t begin = run_begin(total, team, a.p.teams), end = run_begin(total, team + 1, a.p.teams);
  if (L == 0 && t == 0) *a.total = total;
  if (begin >= end) return;
  if (begin < upto && begin >= upto - mine) {
    int64_t at = upto - mine;
    for (int b = b0; b < b1; ++b) {
      const int64_t nb = (int64_t)tiles_of(length_of(a, b)) * a.p.supers;
      if (begin < at + nb) {
        found[0] = b;
        found[1] = begin - at;
        break;
      }
      at += nb;
    }
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane((int)found[0]);
  int64_t within = found[1];
  int64_t left = end - begin;

  // The pieces that this lane loads: piece 64 i + lane of the wavefront's sixteen
  // tokens, in bytes from the first one's address where they lie one after another.
  auto piece_token = [&](int i) { return (8 * i + (lane >> 3)) / (C / 8); };
  auto piece_col = [&](int i) {  // its column in a token, -1 past d_latent or d_rope
    const int tok = piece_token(i), pc = 64 * i + lane - tok * C, col = ((pc & ~7) | ((pc ^ perm(tok)) & 7)) * 8;
    return col < DC ? (col < a.dc ? col : -1) : (col - DC < a.dr ? a.dc + col - DC : -1);
  };
  const bool padded = a.dc != DC || a.dr != kRope;
  const bool rowed = (a.pages == nullptr || a.page_size % 16 == 0) && a.token_stride < (1 << 24);
  uint32_t off[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) off[i] = 2u * (uint32_t)(piece_token(i) * (int)a.token_stride + piece_col(i));
  // what a lane reads of a tile and of P, in bytes
  const int kx = g ^ perm(n);
  const int krow[2] = {((16 * w + n) * C + kx) * 16, ((16 * w + n) * C + (kx ^ 4)) * 16};
  int vrow[NB < 4 ? NB : 4];
#pragma unroll
  for (int k = 0; k < (NB < 4 ? NB : 4); ++k) {
    // lanes 4 r' .. 4 r' + 3 of a group of 16 read token 4 g + r' (and 16 later), 16 columns together
    const int tok = 4 * g + (n >> 2), ch = (w * NB + k) * 2 + ((lane & 3) >> 1);
    vrow[k] = (tok * C + ((ch & ~7) | ((ch ^ perm(tok)) & 7))) * 16 + 8 * (lane & 1);
  }
  const int px = g ^ (n & 7), prow[2] = {n * 128 + px * 16, n * 128 + (px ^ 4) * 16};
  // block 4 w + g of four tokens: step w / 2, place g, half w % 2
  const int pdst = n * 128 + ((4 * (w >> 1) + g) ^ (n & 7)) * 16 + 8 * (w & 1);
  const Lds tiles = lds_of(tile), weights = lds_of(pl);
  // pieces that no load writes are zero in both buffers
  for (int i = t; i < kTile * C; i += kThreads) {
    const u32x4 z = {0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(tile[0])[i] = z;
    reinterpret_cast<u32x4*>(tile[1])[i] = z;
  }
  __syncthreads();

  for (int seg = 0; left > 0; ++seg) {
    const int len = __builtin_amdgcn_readfirstlane(length_of(a, b)), nt = tiles_of(len);
    const int64_t units = (int64_t)nt * a.p.supers;
    if (within >= units) {
      within -= units;
      ++b;
      continue;
    }
    const int super = __builtin_amdgcn_readfirstlane((int)(within / nt)), t0 = __builtin_amdgcn_readfirstlane((int)(within % nt));
    const int t1 = __builtin_amdgcn_readfirstlane((int)(left < nt - t0 ? t0 + left : nt));
    within += t1 - t0;
    left -= t1 - t0;
    const int slot = seg == 0 ? 0 : 1;
    const bool whole = t0 == 0 && t1 == nt;
    if (member == 0 && t == 0) {
      if (t0 == 0) a.first[(int64_t)b * a.p.supers + super] = whole ? -1 : 2 * team + slot;
      if (t1 == nt) a.last[(int64_t)b * a.p.supers + super] = team;
    }
    const int nrow = __builtin_amdgcn_readfirstlane(rows_of(a, b)), r0 = (super * a.p.team + member) * 16 * R;
    if (r0 >= nrow * a.H) continue;
    // query rows' limits: row i of n sees len - n + i + 1 tokens
    const int rlast = min(r0 + 16 * R, nrow * a.H) - 1;
    const int lim_lo = max(len - nrow + r0 / a.H + 1, 0), lim_hi = max(len - nrow + rlast / a.H + 1, 0);
    int lim[R];
    u32x4 qf[R][KS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r0 + 16 * r + n, i = row / a.H, h = row - i * a.H;
      const bool in = row <= rlast;
      lim[r] = in ? max(len - nrow + i + 1, 0) : 0;
      const uint16_t* src = a.q + (int64_t)b * a.qs + (int64_t)i * a.qr + (int64_t)h * a.qh;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int col = 32 * k + 8 * g;
        const int at = col < DC ? (col < a.dc ? col : -1) : (col - DC < a.dr ? a.dc + col - DC : -1);
        qf[r][k] = u32x4{0u, 0u, 0u, 0u};
        if (in && at >= 0) qf[r][k] = *reinterpret_cast<const u32x4*>(src + at);
      }
    }
    f32x4 o[R][NB];
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int k = 0; k < NB; ++k) o[r][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // The address of token `tile * 64 + 16 w + n` of this wavefront's sixteen, and
    // whether any row of the workgroup sees it and its page exists.
    const int32_t* table = a.pages ? a.pages + (int64_t)b * a.pages_stride : nullptr;
    auto page_of = [&](int tl) {
      const int j = tl * kTile + 16 * w + n;
      return j < lim_hi ? (table ? table[j / a.page_size] : b) : -1;
    };
    auto load_tile = [&](int tl, int page, Lds dst) {
      const int j0 = tl * kTile + 16 * w, j = j0 + n;
      const bool ok = page >= 0 && page < a.n_pages;
      const uint32_t valid = (uint32_t)__ballot(ok) & 0xffffu;
      const uint64_t adr = reinterpret_cast<uint64_t>(
          a.cache + (ok ? (int64_t)page * a.page_stride + (int64_t)(j % a.page_size) * a.token_stride : 0));
      const uint32_t alo = (uint32_t)adr, ahi = (uint32_t)(adr >> 32);
      dst += 16 * w * C * 16;
      if (rowed && valid == 0xffffu && !padded) {
        const Global base = (Global)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)ahi) << 32) |
                                     (uint32_t)__builtin_amdgcn_readfirstlane((int)alo));
#pragma unroll
        for (int i = 0; i < NL; ++i) load_lds(base + off[i], dst + 1024 * i);
      } else {
#pragma unroll 1
        for (int i = 0; i < NL; ++i) {
          const int tok = piece_token(i), col = piece_col(i);
          const uint32_t lo = __shfl((int)alo, tok), hi = __shfl((int)ahi, tok);
          if (col >= 0 && (valid >> tok & 1u)) load_lds((Global)(((uint64_t)hi << 32) | lo) + 2 * col, dst + 1024 * i);
        }
      }
      return valid;
    };
    int page = page_of(t0);
    uint32_t valid = load_tile(t0, page, tiles);
    page = t0 + 1 < t1 ? page_of(t0 + 1) : -1;

    for (int tl = t0; tl < t1; ++tl) {
      uint16_t* cur = tile[(tl - t0) & 1];
      const Lds here = tiles + ((tl - t0) & 1) * (kTile * C * 16);
      __builtin_amdgcn_s_waitcnt(0);
      if (valid != 0xffffu) {
        // tokens that no row sees, or of no page, are zero vectors
        for (int i = lane; i < 16 * C; i += 64)
          if (!(valid >> (i / C) & 1u)) reinterpret_cast<u32x4*>(cur)[16 * w * C + i] = u32x4{0u, 0u, 0u, 0u};
      }
      __syncthreads();
      const uint32_t seen = valid;
      if (tl + 1 < t1) {
        valid = load_tile(tl + 1, page, tiles + ((tl - t0 + 1) & 1) * (kTile * C * 16));
        page = tl + 2 < t1 ? page_of(tl + 2) : -1;
      }

      // S^T of this wavefront's sixteen tokens
      f32x4 s[R];
#pragma unroll
      for (int r = 0; r < R; ++r) s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const u32x4 kf = lds_read<u32x4>(here + krow[k & 1] + (k >> 1) * 128);
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = T::mfma(kf, qf[r][k], s[r]);
      }
      // The products' results are taken up here, in the block that made them: the
      // compiler leaves too few wait states before a read behind a branch.
#pragma unroll
      for (int r = 0; r < R; ++r) {
        s[r] *= a.c;
        asm volatile("" : "+v"(s[r]));
      }
      if ((tl + 1) * kTile > lim_lo || seen != 0xffffu) {
        const int j0 = tl * kTile + 16 * w + 4 * g;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[r][i] = j0 + i < lim[r] && (seen >> (4 * g + i) & 1u) ? s[r][i] : -INFINITY;
      }
      const bool edge = (tl + 1) * kTile > lim_lo;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        // a NaN score makes the row's result NaN through its exponential; the maximum passes over it
        float mx = fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3]));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if (g == 0) red[w][16 * r + n] = mx;
      }
      __syncthreads();
      float f[R];
      bool moved = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float mx = m[r];
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, red[i][16 * r + n]);
        const float ref = mx == -INFINITY ? 0.f : mx;
        f[r] = __builtin_amdgcn_exp2f(m[r] - ref);
        moved |= mx != m[r];
        m[r] = mx;
        float p[4], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = __builtin_amdgcn_exp2f(s[r][i] - ref);
          sum += p[i];
        }
        l[r] = mx == -INFINITY ? 0.f : l[r] * f[r] + sum;
        *(__attribute__((address_space(3))) u32x2*)(weights + pdst + 2048 * r) =
            u32x2{T::pack(p[0], p[1]), T::pack(p[2], p[3])};
      }
      // a maximum that moved (seldom, after the first tiles) rescales the rows' sums
      if (__any(moved)) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int k = 0; k < NB; ++k) o[r][k] *= f[r];
      }
      // A token that some rows see and others do not: their weight for it is 0, and 0
      // times an infinity or NaN is not.
      bool odd = false;
      if (edge && lim_lo < lim_hi) {
        bool bad = false;
        const int from = max(lim_lo - tl * kTile, 0), to = min(lim_hi - tl * kTile, kTile);
        for (int i = t; i < (to - from) * DC / 2; i += kThreads) {
          const uint32_t v = reinterpret_cast<const uint32_t*>(cur + (from + i / (DC / 2)) * C * 8)[i % (DC / 2)];
          bad |= (lawless<T>(v) & 0x80008000u) != 0;
        }
        odd = __syncthreads_or(bad);
      } else {
        __syncthreads();
      }
      if (odd) {
        // what the infinities and NaN give to the rows that see them, and zeros in their place
        const int first = tl * kTile, to = min(lim_hi - first, kTile);
#pragma clang loop unroll(disable)
        for (int j = max(lim_lo - first, 0); j < to; ++j) {
          const int blk = j >> 2, at = 4 * (blk >> 3) + (blk & 3), part = 4 * (blk >> 2 & 1) + (j & 3);
#pragma unroll
          for (int k = 0; k < NB; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int ch = (w * NB + k) * 2 + (g >> 1), pc = (ch & ~7) | ((ch ^ perm(j)) & 7);
              uint16_t* at_v = cur + (j * C + pc) * 8 + 4 * (g & 1) + i;
              const uint16_t v = *at_v;
              if ((v & T::kExponent) == T::kExponent) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                  const float p = T::value(pl[(16 * r + n) * kTile + (at ^ (n & 7)) * 8 + part]);
                  if (first + j < lim[r]) o[r][k][i] += p * T::value(v);
                }
              }
            }
        }
        __syncthreads();
        for (int i = t; i < to * DC; i += kThreads) {
          uint16_t* v = cur + (i / DC) * C * 8 + i % DC;
          if (first + i / DC >= lim_lo && (*v & T::kExponent) == T::kExponent) *v = 0;
        }
        __syncthreads();
      }
      // O^T += C^T P^T over the tile's two steps of 32 tokens
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        u32x4 pf[R];
#pragma unroll
        for (int r = 0; r < R; ++r) pf[r] = lds_read<u32x4>(weights + prow[st] + 2048 * r);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          const Lds src = here + vrow[k & 3] + (k >> 2) * 128 + 32 * st * C * 16;
          const u32x2 lo = lds_read_tr(src), hi = lds_read_tr(src + 16 * C * 16);
          const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
          for (int r = 0; r < R; ++r) o[r][k] = T::mfma(vf, pf[r], o[r][k]);
        }
      }
      // wait states for a read of the last results behind the loop's branch
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 7\n\ts_nop 7");
      __builtin_amdgcn_sched_barrier(0);
    }

    // the rows' sums over the lanes and wavefronts that hold their tokens
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] += __shfl_xor(l[r], 16);
      l[r] += __shfl_xor(l[r], 32);
      if (g == 0) red[w][16 * r + n] = l[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r0 + 16 * r + n;
      const float sum = red[0][16 * r + n] + red[1][16 * r + n] + (red[2][16 * r + n] + red[3][16 * r + n]);
      if (whole) {
        if (row > rlast) continue;
        const int i = row / a.H, h = row - i * a.H;
        const float f = sum > 0.f ? 1.f / sum : sum != sum ? NAN : 0.f;
        uint16_t* dst = a.out + (int64_t)b * a.os + (int64_t)i * a.orow + (int64_t)h * a.oh;
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          const int col = (w * NB + k) * 16 + 4 * g;
          if (col < a.dc)
            *reinterpret_cast<u32x2*>(dst + col) = u32x2{T::pack(o[r][k][0] * f, o[r][k][1] * f),
                                                         T::pack(o[r][k][2] * f, o[r][k][3] * f)};
        }
        if (a.lse && w == 0 && g == 0)
          a.lse[((int64_t)b * a.Q + i) * a.H + h] = (m[r] + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        const int64_t at = ((int64_t)L * 2 + slot) * 16 * R + 16 * r + n;
#pragma unroll
        for (int k = 0; k < NB; ++k)
          *reinterpret_cast<f32x4*>(a.part + at * DC + (w * NB + k) * 16 + 4 * g) = o[r][k];
        if (w == 0 && g == 0) a.stat[at] = make_float2(m[r], sum);
      }
    }
    __syncthreads();
  }
}

// The rows of sequences that no run did whole: parts joined against the common
// maximum; rows without a token.  One workgroup a row at a time.
template <class T>
__global__ __launch_bounds__(kThreads) void latent_join_kernel(Args a, int DC) {
  const int t = threadIdx.x, R = a.p.R;
  __shared__ float4 acc[kThreads];
  const int64_t rows = (int64_t)a.B * a.Q * a.H;
  for (int64_t id = blockIdx.x; id < rows; id += gridDim.x) {
    const int b = (int)(id / ((int64_t)a.Q * a.H)), row = (int)(id % ((int64_t)a.Q * a.H)), i = row / a.H, h = row - i * a.H;
    if (i >= rows_of(a, b)) continue;
    uint16_t* dst = a.out + (int64_t)b * a.os + (int64_t)i * a.orow + (int64_t)h * a.oh;
    if (length_of(a, b) == 0) {
      for (int c = t; c < a.dc / 2; c += kThreads) reinterpret_cast<uint32_t*>(dst)[c] = 0u;
      if (a.lse && t == 0) a.lse[id] = -INFINITY;
      continue;
    }
    const int block = row / (16 * R), super = block / a.p.team, member = block % a.p.team;
    const int first = a.first[(int64_t)b * a.p.supers + super];
    if (first < 0) continue;
    const int64_t total = *a.total;
    auto idle = [&](int team) { return run_begin(total, team, a.p.teams) == run_begin(total, team + 1, a.p.teams); };
    const int ta = first >> 1, tb = a.last[(int64_t)b * a.p.supers + super], per = kGroups / 8 / a.p.team;
    auto part_of = [&](int team) {
      const int L = ((team % per) * a.p.team + member) * 8 + team / per;
      return ((int64_t)L * 2 + (team == ta ? first & 1 : 0)) * 16 * R + row % (16 * R);
    };
    float m = -INFINITY;
    for (int k = ta + (t & 63); k <= tb; k += 64)
      if (!idle(k)) m = fmaxf(m, a.stat[part_of(k)].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float ref = m == -INFINITY ? 0.f : m;
    // a quarter or more of the parts to each group of DC / 4 threads
    const int cols = DC / 4, ways = kThreads / cols, way = t / cols, c = t % cols;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    for (int k = ta + way; k <= tb; k += ways) {
      if (idle(k)) continue;
      const int64_t at = part_of(k);
      const float2 st = a.stat[at];
      const float f = __builtin_amdgcn_exp2f(st.x - ref);
      const float4 v = *reinterpret_cast<const float4*>(a.part + at * DC + 4 * c);
      sum += st.y * f;
      o.x += v.x * f;
      o.y += v.y * f;
      o.z += v.z * f;
      o.w += v.w * f;
    }
    __shared__ float sums[8];
    __syncthreads();
    acc[t] = o;
    if (c == 0) sums[way] = sum;
    __syncthreads();
    if (way == 0) {
      for (int k = 1; k < ways; ++k) {
        const float4 v = acc[k * cols + c];
        o.x += v.x;
        o.y += v.y;
        o.z += v.z;
        o.w += v.w;
        sum += sums[k];
      }
      const float f = sum > 0.f ? 1.f / sum : sum != sum ? NAN : 0.f;
      if (4 * c < a.dc)
        *reinterpret_cast<u32x2*>(dst + 4 * c) = u32x2{T::pack(o.x * f, o.y * f), T::pack(o.z * f, o.w * f)};
      if (a.lse && c == 0) a.lse[id] = (m + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

template <class T, int R, int DC>
hipError_t run(const Args& a, hipStream_t s) {
  hipError_t e = launch_timed("latent_attention", latent_kernel<T, R, DC>, dim3(kGroups), dim3(kThreads), s, a);
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)a.B * a.Q * a.H;
  return launch_timed("latent_join", latent_join_kernel<T>, dim3((unsigned)(rows < 2048 ? rows : 2048)), dim3(kThreads),
                      s, a, DC);
}

template <class T>
hipError_t run_type(const Args& a, hipStream_t s) {
  auto by_rows = [&](auto dc) {
    constexpr int DC = decltype(dc)::value;
    return a.p.R == 1 ? run<T, 1, DC>(a, s) : a.p.R == 2 ? run<T, 2, DC>(a, s) : run<T, 4, DC>(a, s);
  };
  return a.dc <= 128   ? by_rows(std::integral_constant<int, 128>{})
         : a.dc <= 256 ? by_rows(std::integral_constant<int, 256>{})
         : a.dc <= 384 ? by_rows(std::integral_constant<int, 384>{})
                       : by_rows(std::integral_constant<int, 512>{});
}

}  // namespace latent
}  // namespace sd
