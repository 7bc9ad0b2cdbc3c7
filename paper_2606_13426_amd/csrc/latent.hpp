// Attention of a few query rows a sequence over a cache of one shared latent
// vector a token (gfx950): keys are the whole vector (latent and rotary part),
// values its latent part.
//
// A workgroup takes 16 R rows (row, head pairs) of one sequence and a run of its
// tokens, 64 at a time.  A tile of the cache enters LDS once and serves both
// products, so a token's bytes come from HBM once for all the rows of a workgroup:
//   S^T [tokens][rows] = C Q^T   a wavefront: 16 or 32 tokens, 16 rows, whose Q stays
//                                in its registers
//   P = 2^{S c - m}, c = scale log2(e); maxima over the tokens' wavefronts by LDS
//   O^T [latent][rows] = C^T P^T a wavefront: a quarter or an eighth of the latent
//                                columns, all rows, accumulators in registers
// on v_mfma_f32_16x16x32.  In both results a lane holds one row of each block of
// 16, so its maximum, sum and rescaling need no exchange inside the products.
// C^T is read by transposing LDS loads; the order in which the 32 tokens of a
// step meet the instruction's k places is the one those loads give, and P is
// stored to match.
//
// m is a reference and not the maximum: it moves when a score exceeds it by more than it
// is allowed to (reach), so the rescaling of O is left out of almost every tile.
// P is rounded to the operands' type, half a step a weight (the instruction takes both
// operands of one type); the weights' sum is of the float32 ones.
//
// Tiles come by loads that write LDS directly, the next one while this one is
// multiplied.  A token's 16-byte pieces are permuted inside each 128 bytes by
// perm(token), which the lanes' global addresses do, so that both products'
// reads meet every bank once.
//
// The tokens of all sequences form one list of tiles that is cut into equal runs,
// one a workgroup (a team of workgroups where one sequence's rows take several: they
// run on one XCD, whose L2 then holds the tile for all of them).  A run may end
// inside a sequence: its part is left in the workspace and joined by
// latent_join_kernel.
//
// With TREE (and fewer rows than latent_wide.hpp is for) the rows of a sequence are nodes of a tree: a row sees the prefix, itself and its
// ancestors.  A node's ancestors are 64 bits, found from the parents by the first wavefront
// of a workgroup whose run reaches behind the prefix, in six doublings (a node's set, joined with that
// of the node its chain of parents has reached so far), and kept in LDS beside the
// rows; only tiles behind the prefix look at them.
//
// What bounds it, on MI355X.  Up to 32 rows: the cache's stream (2 sequences of 131072
// tokens, 32 heads, bf16: 59 us, 5.1 TB/s, and 13 us for the join of 128 parts a row).
// With 64 rows the phases between a tile's three barriers: one workgroup fills a compute
// unit's LDS, LDS is read in 40 % of the cycles, the matrix cores are busy in 26 %, vector
// instructions issue in 22 %, and wavefronts wait for 42 % of their time (64 ragged
// sequences of up to 6000 tokens, 128 heads: 122 us, 2.2 TB/s, 0.5 PFLOP/s; a tile takes
// 3800 cycles, a run's first tile and Q 16000, its stores 9000).
// Wavefronts of 32 rows, which read K from LDS twice a tile instead of four times, were slower
// (155 us where these took 130): with Q in registers there is room for fewer operands ahead of the products.
// A short sequence is latency: 15 us for 777 tokens, 5 for the join.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "latent_common.hpp"

namespace sd {
namespace latent {

constexpr int kGroups = 256;  // workgroups: one a compute unit (the tiles fill its LDS)

// How the rows of a sequence are dealt to workgroups: blocks of 16 R rows, teams
// of `team` blocks that walk the same tokens (up to four, so that a tile's second to
// fourth reader finds it in the XCD's L2), `supers` teams' worth a sequence.
struct Plan {
  int R, blocks, team, supers, teams;
};
inline int most_r(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }
inline Plan plan_of(int64_t rows, int R) {
  Plan p;
  p.R = R;
  p.blocks = (int)((rows + 16 * p.R - 1) / (16 * p.R));
  p.team = p.blocks % 4 == 0 ? 4 : p.blocks % 2 == 0 ? 2 : p.blocks == 3 ? 3 : 1;
  p.supers = p.blocks / p.team;
  p.teams = 8 * (kGroups / 8 / p.team);
  return p;
}
// Many rows a workgroup read the cache less often, few leave smaller parts to join.  By the
// tiles of 64 rows and 64 tokens that a compute unit has if every sequence is as long as its
// pages allow (the lengths are on the device: short sequences under a wide table get the rows of
// long ones, in the first line 25 us for 20); in us (both kernels) with R = 1 / 2 / 4, H heads of one row each:
//   1 x 800 tokens, H = 64, 0.05 tiles:  20 / 21 / 25     4 x 4000, H = 128, 2:    41 / 40 / 46
//   1 x 4000, H = 128, 0.5:              29 / 31 / 34     16 x 4000, H = 128, 8:   83 / 62 / 61
//   8 x 4000, H = 64, 2:                 41 / 40 / 47     64 x 4000, H = 64, 16:   147 / 105 / 94
inline Plan plan(int B, int Q, int H, int capacity) {
  const int64_t rows = (int64_t)Q * H, tiles = ((int64_t)capacity + kTile - 1) / kTile * B * ((rows + 63) / 64);
  const int most = most_r(rows);
  return plan_of(rows, tiles < kGroups ? 1 : tiles < 8 * kGroups && most > 2 ? 2 : most);
}

// The kernel of 128 rows a workgroup (latent_wide.hpp), for trees: by its tiles of 128 rows and 64 tokens, 12 a
// compute unit where sequences are cut (its parts to join are twice as large), 2 where there is a block of rows for
// most compute units and mostly done whole.  In us (all kernels), at most 64 rows a workgroup / 128:
//   1 tree of 64 nodes, 16 heads, 6400 tokens, 3.1 tiles a unit:  53 / 59    25600, 12.5: 99 / 93     100000, 49: 293 / 227
//   64 trees of 16 nodes, 16 heads, 1600 tokens, 12.5:            94 / 108   3200, 25:    161 / 161   6400, 50:   304 / 263
//   24 trees of 20 nodes, 32 heads (120 blocks), 400 tokens, 3.3: 63 / 57    1600, 11.7:  107 / 103   6400, 47:   303 / 259
//   8 trees of 32 nodes, 128 heads (256 blocks), 100 tokens, 2:   64 / 50    6400, 100:   575 / 423
//   30 trees of up to 46 nodes, 16 heads (180 blocks), up to 383 tokens, 4.2:  66 / 57
constexpr int kWideRows = 128, kWideR = kWideRows / 16;
inline bool wide_fits(int64_t rows, int dc, int dr) { return rows >= kWideRows && dc == 512 && dr == kRope; }
inline Plan tree_plan(int B, int Q, int H, int dc, int dr, int capacity) {
  const int64_t rows = (int64_t)Q * H, blocks = (rows + kWideRows - 1) / kWideRows * B;
  const int64_t tiles = ((int64_t)capacity + kTile - 1) / kTile * blocks;
  const bool many = tiles >= 12 * kGroups || (blocks >= kGroups * 5 / 8 && tiles >= 2 * kGroups);
  return many && wide_fits(rows, dc, dr) ? plan_of(rows, kWideR) : plan(B, Q, H, capacity);
}

struct Args {
  int B, Q, H, dc, dr;
  float c;        // |scale| log2(e)
  uint32_t flip;  // sign bits of a pair, to negate q where scale is negative
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
  float2* stat;    // [kGroups][2][16 R] (reference in log2 units, sum)
  int32_t* first;  // [B][supers] 2 team + slot of the run that starts the sequence; -1: one run did it all
  int32_t* last;   // [B][supers] the team that ends it
  const int32_t* parents;  // [B][Q], with TREE
};

__device__ __forceinline__ int length_of(const Args& a, int b) { return min(max(load_global<int32_t>(a.lens + b), 0), a.capacity); }
__device__ __forceinline__ int rows_of(const Args& a, int b) {
  return a.rows ? min(max(load_global<int32_t>(a.rows + b), 0), a.Q) : a.Q;
}
__device__ __forceinline__ int tiles_of(int len) { return (len + kTile - 1) / kTile; }
// Team `team` of `teams` (a multiple of 8 that go round the XCDs) runs as workgroups group_of(.., 0..).
__device__ __forceinline__ int group_of(int team, int member, int size) {
  return (team / 8 * size + member) * 8 + team % 8;
}

// The nodes that node `lane` of sequence b sees, itself among them; up: its parent in the tree.
__device__ __forceinline__ uint64_t ancestors(int up, int lane) {
  uint64_t set = 1ull << lane;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const int from = up < 0 ? lane : up;
    const uint64_t more = (uint64_t)__shfl((unsigned long long)set, from);
    const int next = __shfl(up, from);
    set |= more;
    up = up < 0 ? -1 : next;
  }
  return set;
}

template <class T, int R, int DC, bool TREE>
__global__ __launch_bounds__(R == 1 ? 256 : 512) void latent_kernel(Args a) {
  constexpr int kWaves = R == 1 ? 4 : 8, kLanes = 64 * kWaves;
  constexpr int WR = R, WT = kWaves / WR, TB = kTile / 16 / WT;  // row groups of 16, token groups of 16 TB
  constexpr int C = (DC + kRope) / 8;     // 16-byte pieces of a token
  constexpr int KS = (DC + kRope) / 32;   // steps of 32 columns of Q
  constexpr int NB = DC / (16 * kWaves);  // blocks of 16 latent columns of a wavefront
  constexpr int TW = kTile / kWaves;      // tokens that a wavefront loads
  constexpr int NL = TW * C / 64;         // its loads, of 64 pieces
  constexpr int NV = NB < 4 ? NB : 4;
  static_assert(C % 8 == 0 && DC % 128 == 0 && NL * 64 == TW * C, "whole 128-byte segments, blocks and loads");
  __shared__ __align__(16) uint16_t tile[2][kTile * C * 8];
  __shared__ __align__(16) uint16_t pl[16 * R * kTile];
  __shared__ float red[WT][16 * R];
  __shared__ float fac[16 * R];
  __shared__ int limits[16 * R];
  __shared__ uint64_t kin[TREE ? 16 * R : 1];  // a row's node and its ancestors
  __shared__ int moved[2][WR + 1];  // whose rows' reference moved; last: values that are no numbers
  __shared__ uint32_t present[kWaves];

  const int t = threadIdx.x, lane = t & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6), wt = w % WT, wr = w / WT;
  const int L = blockIdx.x, i8 = L / 8, team = i8 / a.p.team * 8 + L % 8, member = i8 % a.p.team;

  // this team's run of the list of all sequences' tiles: found by each wavefront for itself, in blocks
  // of 64 sequences, the first of which stays in registers
  auto tiles_at = [&](int len, int bb) { return bb < a.B ? tiles_of(len) * a.p.supers : 0; };
  auto scan = [&](int v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(v, d);
      if (lane >= d) v += o;
    }
    return v;
  };
  const int len0 = length_of(a, min(lane, a.B - 1)), tiles0 = tiles_at(len0, lane), upto0 = scan(tiles0);
  int total = __builtin_amdgcn_readlane(upto0, 63);
  for (int b0 = 64; b0 < a.B; b0 += 64)
    total += __builtin_amdgcn_readlane(scan(tiles_at(length_of(a, min(b0 + lane, a.B - 1)), b0 + lane)), 63);
  const int teams = min(a.p.teams, total);
  if (team >= teams) return;
  const int share = total / teams, more = total - share * teams;
  const int begin = team * share + min(team, more);
  int left = share + (team < more ? 1 : 0);
  int b = 0, within = 0;
  for (int b0 = 0, at = 0;; b0 += 64) {
    const int mine = b0 == 0 ? tiles0 : tiles_at(length_of(a, min(b0 + lane, a.B - 1)), b0 + lane);
    const int upto = b0 == 0 ? upto0 : scan(mine);
    const uint64_t hit = __ballot(at + upto > begin);
    if (hit) {
      const int i = __ffsll((unsigned long long)hit) - 1;
      b = b0 + i;
      within = begin - at - __builtin_amdgcn_readlane(upto - mine, i);
      break;
    }
    at += __builtin_amdgcn_readlane(upto, 63);
    if (b0 + 64 >= a.B) return;  // (not reached: begin is below the total)
  }

  // The pieces that this lane loads: piece 64 i + lane of the wavefront's TW tokens.
  auto piece_token = [&](int i, int ln) { return (8 * i + (ln >> 3)) / (C / 8); };
  auto piece_col = [&](int i, int ln) {  // its column in a token, -1 past d_latent or d_rope
    const int tok = piece_token(i, ln), pc = 64 * i + ln - tok * C, col = ((pc & ~7) | ((pc ^ perm(tok)) & 7)) * 8;
    return col < DC ? (col < a.dc ? col : -1) : (col - DC < a.dr ? a.dc + col - DC : -1);
  };
  // The lane, for the loop's rare paths: what they compute from it is not kept in registers through
  // the others.
  auto rare = [&](int v) {
    asm volatile("" : "+v"(v));
    return v;
  };
  const bool padded = a.dc != DC || a.dr != kRope;
  // Where a wavefront's tokens lie one after another in one page, a tile's loads have one scalar
  // address and a lane's fixed offsets.
  const bool rowed = a.token_stride < (1 << 24);
  // The same of a sequence's rows of Q, heads side by side in every one (16 rows would be one wavefront's
  // then: 17 us instead of 15 for a short sequence).
  const bool level = R > 1 && (a.Q == 1 || a.qr == a.H * a.qh) && a.qh < (1 << 24) && rowed;
  uint32_t off[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    // (a column that is not there lies past every view's end: nothing is read for it)
    const int col = piece_col(i, lane);
    off[i] = col < 0 ? 0x80000000u : 2u * (uint32_t)(piece_token(i, lane) * (int)a.token_stride + col);
  }
  // what a lane reads of a tile and of P, in bytes
  const int kx = g ^ perm(n);
  const int krow[2] = {((16 * TB * wt + n) * C + kx) * 16, ((16 * TB * wt + n) * C + (kx ^ 4)) * 16};
  int vrow[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    // lanes 4 r' .. 4 r' + 3 of a group of 16 read token 4 g + r' (and 16 later), 16 columns together
    const int tok = 4 * g + (n >> 2), ch = (w * NB + k) * 2 + ((lane & 3) >> 1);
    vrow[k] = (tok * C + ((ch & ~7) | ((ch ^ perm(tok)) & 7))) * 16 + 8 * (lane & 1);
  }
  const int px = g ^ (n & 7), prow[2] = {n * 128 + px * 16, n * 128 + (px ^ 4) * 16};
  // four tokens 4 g of 16-token block v = TB wt + j: step v / 2, place g, half v % 2
  int pdst[TB];
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int v = TB * wt + j;
    pdst[j] = n * 128 + ((4 * (v >> 1) + g) ^ (n & 7)) * 16 + 8 * (v & 1) + 2048 * wr;
  }
  const Lds tiles = lds_of(tile), weights = lds_of(pl);

  if (padded) {
    // pieces that no load writes are zero in both buffers
    for (int i = t; i < 2 * kTile * C; i += kLanes) reinterpret_cast<u32x4*>(tile)[i] = u32x4{0u, 0u, 0u, 0u};
  }
  __syncthreads();

  for (int seg = 0; left > 0; ++seg) {
    const int len = b < 64 ? __builtin_amdgcn_readlane(len0, b) : __builtin_amdgcn_readfirstlane(length_of(a, b)), nt = tiles_of(len), units = nt * a.p.supers;
    if (within >= units) {
      within -= units;
      ++b;
      --seg;
      continue;
    }
    const int super = within / nt, t0 = within - super * nt, t1 = min(t0 + left, nt);
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
    // (a tree's rows all see the prefix; what they see of the rest their nodes say)
    const int lim_lo = TREE ? max(len - nrow, 0) : max(len - nrow + r0 / a.H + 1, 0), lim_hi = max(len - nrow + rlast / a.H + 1, 0);
    [[maybe_unused]] int up = -1;
    if constexpr (TREE) {
      if (w == 0 && t1 * kTile > lim_lo && lane < nrow) up = load_global<int32_t>(a.parents + (int64_t)b * a.Q + lane);
    }

    // Tile tl's part of this wavefront: tokens tl * 64 + TW w .. + TW - 1.  Returns which of them some
    // row sees and whose page exists; the others are not loaded.
    const int32_t* table = a.pages ? a.pages + (int64_t)b * a.pages_stride : nullptr;
    // (the page of a whole tile's part is asked for a tile ahead: it would be waited for)
    auto page_of = [&](int tl) {
      const int j0 = tl * kTile + TW * w;
      return table && rowed && j0 < lim_hi ? load_global<int32_t>(table + j0 / a.page_size) : b;
    };
    // What a tile's loads need; `on` says that they go by the view, one after another (next_load), and
    // valid which tokens they bring.  Tiles of another kind are loaded here.
    struct Load {
      u32x4 view;
      uint32_t dst, valid;
      uint64_t on;
    };
    auto start_load = [&](int tl, int ahead, Lds dst) -> Load {
      Load ld{u32x4{0u, 0u, 0u, 0u}, 0u, 0u, 0ull};
      const int j0 = tl * kTile + TW * w, count = min(max(lim_hi - j0, 0), TW);
      dst += TW * w * C * 16;
      const int pg0 = table ? j0 / a.page_size : 0, in = j0 - pg0 * a.page_size;
      if (rowed && count == TW && (!table || in + TW <= a.page_size)) {
        const int page = __builtin_amdgcn_readfirstlane(ahead);
        if (page < 0 || page >= a.n_pages) return ld;
        ld.view = lds_view(a.cache + (int64_t)page * a.page_stride + (int64_t)in * a.token_stride,
                           2 * ((TW - 1) * a.token_stride + a.dc + a.dr));
        ld.dst = lds_address(dst);
        ld.valid = (1u << TW) - 1u;
        ld.on = ~0ull;
        return ld;
      }
      const int ln = rare(lane), j = j0 + ln % TW, pg = j / a.page_size;
      const int page = ln % TW < count ? (table ? load_global<int32_t>(table + pg) : b) : -1;
      const bool ok = page >= 0 && page < a.n_pages;
      const uint32_t valid = (uint32_t)__ballot(ok) & ((1u << TW) - 1u);
      const uint64_t adr = reinterpret_cast<uint64_t>(
          a.cache + (ok ? (int64_t)page * a.page_stride + (int64_t)(table ? j - pg * a.page_size : j) * a.token_stride : 0));
#pragma unroll 1
      for (int i = 0; i < NL; ++i) {
        const int tok = piece_token(i, ln), col = piece_col(i, ln);
        const uint32_t lo = __shfl((int)(uint32_t)adr, tok), hi = __shfl((int)(uint32_t)(adr >> 32), tok);
        if (col >= 0 && (valid >> tok & 1u)) load_lds((Global)(((uint64_t)hi << 32) | lo) + 2 * col, dst + 1024 * i);
      }
      ld.valid = valid;
      return ld;
    };
    // tokens that no row sees, or of no page, become zero vectors
    auto clear_rest = [&](uint32_t valid, Lds dst) {
      dst += TW * w * C * 16;
      for (int i = rare(lane); i < TW * C; i += 64)
        if (!(valid >> (i / C) & 1u)) *(__attribute__((address_space(3))) u32x4*)(dst + 16 * i) = u32x4{0u, 0u, 0u, 0u};
    };
    int next = t0 + 1 < t1 ? page_of(t0 + 1) : 0;
    // Q's rows come like a tile, into the other buffer, in whole lines and once a workgroup, and from
    // there into registers (each lane's own 16 bytes straight from memory: 131 us instead of 123 for 64
    // sequences of up to 6000 tokens, 128 heads).
    const Lds held = tiles + kTile * C * 16;
    uint32_t valid;
    {
      const Load ld = start_load(t0, page_of(t0), tiles);
      valid = ld.valid;
      const uint16_t* src = a.q + (int64_t)b * a.qs;
      if (level) {
        // a wavefront's rows as it loads tokens; those past the last come as zeros
        const int from = r0 + TW * w, have = min(rlast + 1 - from, 16 * R - TW * w);
        const u32x4 view = lds_view(src + (int64_t)from * a.qh, have > 0 ? 2 * ((have - 1) * a.qh + a.dc + a.dr) : 0);
        const uint32_t to = lds_address(held + TW * w * C * 16), more = 2u * (uint32_t)(int)(a.qh - a.token_stride);
        if (TW * w < 16 * R)
          each<NL>([&](auto i) {
            load_lds_view<1024 * decltype(i)::value>(view, off[i] + more * (uint32_t)piece_token(i, lane), to, ~0ull);
          });
      } else {
#pragma unroll 1
        for (int s = 64 * w; s < 16 * R * C; s += kLanes) {
          const int ln = rare(lane), piece = s + ln, row = piece / C, pc = piece - row * C;
          const int col = ((pc & ~7) | ((pc ^ perm(row)) & 7)) * 8;
          const int at = col < DC ? (col < a.dc ? col : -1) : (col - DC < a.dr ? a.dc + col - DC : -1);
          const int own = min(r0 + row, rlast), i = own / a.H, h = own - i * a.H;
          if (at >= 0) load_lds((Global)(src + (int64_t)i * a.qr + (int64_t)h * a.qh + at), held + 16 * s);
        }
      }
      each<NL>([&](auto i) { load_lds_view<1024 * decltype(i)::value>(ld.view, off[i], ld.dst, ld.on); });
      if (ld.on)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");  // Q is there, the tile on its way
      else
        __builtin_amdgcn_s_waitcnt(0);
    }
    if (t < 2 * (WR + 1)) moved[t / (WR + 1)][t % (WR + 1)] = 0;
    if constexpr (TREE) {
      if (w == 0 && t1 * kTile > lim_lo) {
        const uint64_t set = ancestors(up < lane ? up : -1, lane);
        const uint64_t mine = (uint64_t)__shfl((unsigned long long)set, min(r0 + lane, rlast) / a.H);
        if (lane < 16 * R) kin[lane] = mine;
      }
    } else {
      if (t < 16 * R) limits[t] = r0 + t <= rlast ? len - nrow + (r0 + t) / a.H + 1 : 0;
    }
    lds_barrier();

    u32x4 qf[KS];
    const int row = r0 + 16 * wr + n, lim = row <= rlast ? max(len - nrow + row / a.H + 1, 0) : 0;
#pragma unroll
    for (int k = 0; k < KS; ++k)
      qf[k] = lds_read<u32x4>(held + ((16 * wr + n) * C + (k & 1 ? kx ^ 4 : kx)) * 16 + (k >> 1) * 128) ^ a.flip;
    f32x4 o[R][NB];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < NB; ++k) o[r][k] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int tl = t0; tl < t1; ++tl) {
      uint16_t* cur = tile[(tl - t0) & 1];
      const Lds here = tiles + ((tl - t0) & 1) * (kTile * C * 16);
      __builtin_amdgcn_s_waitcnt(0);
      if (valid != (1u << TW) - 1u) clear_rest(valid, here);
      if (lane == 0) present[w] = valid;
      __syncthreads();
      if (t <= WR) moved[(tl - t0 + 1) & 1][t] = 0;
      Load ld{u32x4{0u, 0u, 0u, 0u}, 0u, 0u, 0ull};
      if (tl + 1 < t1) {
        const int page = next;
        if (tl + 2 < t1) next = page_of(tl + 2);
        ld = start_load(tl + 1, page, tiles + ((tl - t0 + 1) & 1) * (kTile * C * 16));
        valid = ld.valid;
      }
      // the scalar registers of a uniform value that a branch chose
      ld.view = u32x4{uniform(ld.view[0]), uniform(ld.view[1]), uniform(ld.view[2]), kBufferWord3};
      ld.dst = uniform(ld.dst);
      ld.on = (uint64_t)0 - (uint64_t)(uniform((uint32_t)ld.on) & 1u);

      f32x4 s[TB];
#pragma unroll
      for (int j = 0; j < TB; ++j) s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      {
        // Two steps' pieces are read while the two before are multiplied.  The next tile's loads go out
        // between them: a load of 1 KB takes the unit that makes its addresses 16 cycles, so that
        // 72 in a row would hold up the wavefronts for longer than the products take.
        u32x4 kf[2][2][TB];
        auto read = [&](int k) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
              kf[(k >> 1) & 1][i][j] = lds_read<u32x4>(here + krow[i] + (k >> 1) * 128 + 16 * j * C * 16);
        };
        read(0);
        each<KS / 2>([&](auto step) {
          constexpr int h = decltype(step)::value, k = 2 * h;
          if (k + 2 < KS) read(k + 2);
          __builtin_amdgcn_sched_barrier(0);
          each<NL>([&](auto i) {
            if constexpr (i * (KS / 2) / NL == h) load_lds_view<1024 * decltype(i)::value>(ld.view, off[i], ld.dst, ld.on);
          });
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) s[j] = T::mfma(kf[h & 1][i][j], qf[k + i], s[j]);
          __builtin_amdgcn_sched_barrier(0);
        });
      }
      // The products' results are taken up here, in the block that made them: the
      // compiler leaves too few wait states before a read behind a branch.
#pragma unroll
      for (int j = 0; j < TB; ++j) asm volatile("" : "+v"(s[j]));
      // which of the wavefront's tokens are there, TW bits from each that loaded them
      constexpr int kFrom = 16 * TB / TW;
      uint32_t seen = 0;
#pragma unroll
      for (int j = 0; j < kFrom; ++j) seen |= present[kFrom * wt + j] << (TW * j);
      seen = (uint32_t)__builtin_amdgcn_readfirstlane((int)seen);
      const bool edge = (tl + 1) * kTile > lim_lo;
      if (edge || seen != (uint32_t)((1ull << (16 * TB)) - 1)) {
        const int ahead = lim - (tl * kTile + 16 * TB * wt + 4 * g);  // its tokens from this lane's first on
        uint32_t have = seen >> (4 * g);
        if constexpr (TREE) {
          if (edge) {
            const int ln = rare(lane);
            const uint64_t set = kin[16 * wr + (ln & 15)];
            const int node = tl * kTile + 16 * TB * wt + 4 * (ln >> 4) - (len - nrow);  // of this lane's first token
            have &= node >= 64   ? 0u
                    : node >= 0  ? (uint32_t)(set >> node)
                    : node > -32 ? ((uint32_t)set << -node) | ((1u << -node) - 1u)
                                 : ~0u;
          }
        }
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[j][i] = 16 * j + i < ahead && (have & (1u << (16 * j + i))) ? s[j][i] : -INFINITY;
      }
      // a NaN score makes the row's result NaN through its exponential; the maximum passes over it
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < TB; ++j) mx = fmaxf(mx, fmaxf(fmaxf(s[j][0], s[j][1]), fmaxf(s[j][2], s[j][3])));
      mx = quarter_max(mx);
      if (g == 0) red[wt][16 * wr + n] = mx;
      lds_barrier();
#pragma unroll
      for (int j = 0; j < WT; ++j) mx = fmaxf(mx, red[j][16 * wr + n]);
      mx *= a.c;
      if (const bool up = mx > reach<T>(m); __any(up)) {
        const float to = up ? reference<T>(mx) : m, f = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= f;
        if (wt == 0 && g == 0) fac[16 * wr + n] = f;
        if (wt == 0) moved[(tl - t0) & 1][wr] = 1;
      }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(__fmaf_rn(s[j][i], a.c, -ref));
        l += (p[0] + p[1]) + (p[2] + p[3]);
        *(__attribute__((address_space(3))) u32x2*)(weights + pdst[j]) = u32x2{T::pack(p[0], p[1]), T::pack(p[2], p[3])};
      }
      // A token that some rows see and others do not: their weight for it is 0, and 0
      // times an infinity or NaN is not.
      if (edge && lim_lo < lim_hi) {
        uint32_t bad = 0;
        const int from = max(lim_lo - tl * kTile, 0), to_j = min(lim_hi - tl * kTile, kTile);
        for (int i = rare(t); i < (to_j - from) * DC / 2; i += kLanes)
          bad |= lawless<T>(reinterpret_cast<const uint32_t*>(cur + (from + i / (DC / 2)) * C * 8)[i % (DC / 2)]);
        if (__any((bad & 0x80008000u) != 0) && lane == 0) moved[(tl - t0) & 1][WR] = 1;
      }
      lds_barrier();
#pragma unroll
      for (int q = 0; q < WR; ++q)
        if (__builtin_amdgcn_readfirstlane(moved[(tl - t0) & 1][q])) {
#pragma unroll
          for (int k = 0; k < NB; ++k) o[q][k] *= fac[16 * q + n];
        }
      if (__builtin_amdgcn_readfirstlane(moved[(tl - t0) & 1][WR])) {
        // what the infinities and NaN give to the rows that see them, and zeros in their place
        const int first = tl * kTile, to_j = min(lim_hi - first, kTile), ln = rare(lane), ng = ln >> 4, nn = ln & 15;
#pragma clang loop unroll(disable)
        for (int j = max(lim_lo - first, 0); j < to_j; ++j) {
          const int blk = j >> 2, at = 4 * (blk >> 3) + (blk & 3), part = 4 * (blk >> 2 & 1) + (j & 3);
#pragma unroll
          for (int k = 0; k < NB; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int ch = (w * NB + k) * 2 + (ng >> 1), pc = (ch & ~7) | ((ch ^ perm(j)) & 7);
              const uint16_t v = cur[(j * C + pc) * 8 + 4 * (ng & 1) + i];
              if ((v & T::kExponent) == T::kExponent) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                  const float p = T::value(pl[(16 * r + nn) * kTile + (at ^ (nn & 7)) * 8 + part]);
                  if constexpr (TREE) {
                    const int node = first + j - (len - nrow);  // (in [0, 64): from the prefix's end to the last row's)
                    if (kin[16 * r + nn] >> node & 1u) o[r][k][i] += p * T::value(v);
                  } else {
                    if (first + j < limits[16 * r + nn]) o[r][k][i] += p * T::value(v);
                  }
                }
              }
            }
        }
        __syncthreads();
        for (int i = rare(t); i < to_j * DC; i += kLanes) {
          uint16_t* v = cur + (i / DC) * C * 8 + i % DC;
          if (first + i / DC >= lim_lo && (*v & T::kExponent) == T::kExponent) *v = 0;
        }
        __syncthreads();
      }
      // O^T += C^T P^T over the tile's two steps of 32 tokens; the next block's values are read while
      // one is multiplied
      {
        u32x4 pf[R], vf[2];
        auto read = [&](int i) {
          const Lds src = here + vrow[i % NB & 3] + (i % NB >> 2) * 128 + 32 * (i / NB) * C * 16;
          const u32x2 lo = lds_read_tr(src), hi = lds_read_tr(src + 16 * C * 16);
          vf[i & 1] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        };
        read(0);
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
          if (i % NB == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) pf[r] = lds_read<u32x4>(weights + prow[i / NB] + 2048 * r);
          }
          if (i + 1 < 2 * NB) read(i + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int r = 0; r < R; ++r) o[r][i % NB] = T::mfma(vf[i & 1], pf[r], o[r][i % NB]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      // wait states for a read of the last results behind the loop's branch
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 7\n\ts_nop 7");
      __builtin_amdgcn_sched_barrier(0);
    }

    // the rows' sums over the lanes and wavefronts that hold their tokens
    __syncthreads();
    l = quarter_sum(l);
    if (g == 0) red[wt][16 * wr + n] = l;
    if (g == 0 && wt == 0) fac[16 * wr + n] = m;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r0 + 16 * r + n;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < WT; ++j) sum += red[j][16 * r + n];
      const float ref = fac[16 * r + n];
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
          a.lse[((int64_t)b * a.Q + i) * a.H + h] = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        const int64_t at = ((int64_t)L * 2 + slot) * 16 * R + 16 * r + n;
#pragma unroll
        for (int k = 0; k < NB; ++k)
          *reinterpret_cast<f32x4*>(a.part + at * DC + (w * NB + k) * 16 + 4 * g) = o[r][k];
        if (w == 0 && g == 0) a.stat[at] = make_float2(ref, sum);
      }
    }
    __syncthreads();
  }
}

// The rows of sequences that no run did whole: parts joined against the largest
// reference; rows without a token.  With WAYS = 1 a wavefront takes a row; with WAYS =
// 4, for rows of many parts, the four of a workgroup take the parts of 128 columns of a
// row in turn.
template <class T, int DC, int WAYS>
__global__ __launch_bounds__(kThreads) void latent_join_kernel(Args a) {
  constexpr int NC = WAYS == 1 ? DC / 128 : 1;   // pairs of columns of a lane
  constexpr int CH = WAYS == 1 ? 1 : DC / 128;   // wavefronts that share a row by columns
  __shared__ float2 acc[4][64];
  __shared__ float sums[4];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int way = WAYS == 1 ? 0 : w, per_group = 4 / WAYS;
  const int rows = a.B * a.Q * a.H, R = a.p.R;  // (times DC / 128 below 2^31: the rows have an output each)
  for (int base = blockIdx.x * per_group; base < rows * CH; base += gridDim.x * per_group) {
    const int unit = base + (WAYS == 1 ? w : 0), id = unit / CH, col0 = unit % CH * 128 + 2 * lane;
    if (id >= rows) break;
    const int b = id / (a.Q * a.H), row = id - b * a.Q * a.H, i = row / a.H, h = row - i * a.H;
    if (i >= rows_of(a, b)) continue;
    uint16_t* dst = a.out + (int64_t)b * a.os + (int64_t)i * a.orow + (int64_t)h * a.oh;
    const bool says = a.lse && way == 0 && lane == 0 && unit % CH == 0;
    if (length_of(a, b) == 0) {
#pragma unroll
      for (int k = 0; k < NC; ++k)
        if (way == 0 && col0 + 128 * k < a.dc) *reinterpret_cast<uint32_t*>(dst + col0 + 128 * k) = 0u;
      if (says) a.lse[id] = -INFINITY;
      continue;
    }
    const int block = row / (16 * R), super = block / a.p.team, member = block - super * a.p.team;
    const int first = a.first[(int64_t)b * a.p.supers + super];
    if (first < 0) continue;
    const int ta = first >> 1, tb = a.last[(int64_t)b * a.p.supers + super];
    auto part_of = [&](int team) {
      return (group_of(team, member, a.p.team) * 2 + (team == ta ? first & 1 : 0)) * 16 * R + row % (16 * R);
    };
    float m = -INFINITY;
    for (int k = ta + lane; k <= tb; k += 64) m = fmaxf(m, a.stat[part_of(k)].x);
    m = across(m, true, true);
    m = across(m, false, true);
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float ref = m == -INFINITY ? 0.f : m;
    float2 o[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) o[k] = make_float2(0.f, 0.f);
    float sum = 0.f;
    for (int k0 = ta + way; k0 <= tb; k0 += 64 * WAYS) {
      // lane j: the weight and place of part k0 + WAYS j
      const int mine = k0 + WAYS * lane, at = mine <= tb ? part_of(mine) : 0;
      const float2 st = mine <= tb ? a.stat[at] : make_float2(-INFINITY, 0.f);
      const float f = __builtin_amdgcn_exp2f(st.x - ref);
      sum += mine <= tb ? st.y * f : 0.f;
      const int count = min((tb - k0) / WAYS + 1, 64);
#pragma unroll(WAYS == 1 ? 4 : 16)
      for (int j = 0; j < count; ++j) {
        const float fj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), j));
        const float* src = a.part + (int64_t)__builtin_amdgcn_readlane(at, j) * DC + col0;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          const float2 v = *reinterpret_cast<const float2*>(src + 128 * k);
          o[k].x = __fmaf_rn(v.x, fj, o[k].x);
          o[k].y = __fmaf_rn(v.y, fj, o[k].y);
        }
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (WAYS > 1) {
      __syncthreads();
      acc[way][lane] = o[0];
      if (lane == 0) sums[way] = sum;
      __syncthreads();
      if (way > 0) continue;
      sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
      for (int q = 1; q < WAYS; ++q) {
        o[0].x += acc[q][lane].x;
        o[0].y += acc[q][lane].y;
      }
    }
    const float f = sum > 0.f ? 1.f / sum : sum != sum ? NAN : 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k)
      if (col0 + 128 * k < a.dc)
        *reinterpret_cast<uint32_t*>(dst + col0 + 128 * k) = T::pack(o[k].x * f, o[k].y * f);
    if (says) a.lse[id] = (m + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

// One wavefront a row, or four for 128 columns of it where rows are few and may have eight parts or
// more.  In us, one / four: 64 rows of 128 parts 40 / 13, 512 rows of 16 parts 9.7 / 9.6, 2048
// rows of 4 parts 7 / 21, 8192 rows of 2 parts 13 / 67.
template <class T, int DC>
hipError_t join(const Args& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.Q * a.H, many = rows * (DC / 128), few = (rows + 3) / 4;
  return rows < 1024 && a.p.teams >= 8 * (int64_t)a.B * a.p.supers
             ? launch_timed("latent_join", latent_join_kernel<T, DC, 4>, dim3((unsigned)(many < 4096 ? many : 4096)),
                            dim3(kThreads), s, a)
             : launch_timed("latent_join", latent_join_kernel<T, DC, 1>, dim3((unsigned)(few < 4096 ? few : 4096)),
                            dim3(kThreads), s, a);
}

template <class T, int R, int DC, bool TREE>
hipError_t run(const Args& a, hipStream_t s) {
  const hipError_t e = launch_timed(TREE ? "latent_tree" : "latent_attention", latent_kernel<T, R, DC, TREE>, dim3(kGroups),
                                    dim3(R == 1 ? 256 : 512), s, a);
  return e != hipSuccess ? e : join<T, DC>(a, s);
}

template <class T, bool TREE = false>
hipError_t run_type(const Args& a, hipStream_t s) {
  auto by_rows = [&](auto dc) {
    constexpr int DC = decltype(dc)::value;
    return a.p.R == 1 ? run<T, 1, DC, TREE>(a, s) : a.p.R == 2 ? run<T, 2, DC, TREE>(a, s) : run<T, 4, DC, TREE>(a, s);
  };
  return a.dc <= 128   ? by_rows(std::integral_constant<int, 128>{})
         : a.dc <= 256 ? by_rows(std::integral_constant<int, 256>{})
         : a.dc <= 384 ? by_rows(std::integral_constant<int, 384>{})
                       : by_rows(std::integral_constant<int, 512>{});
}

}  // namespace latent
}  // namespace sd
