// Attention of many rows a sequence over a cache of one shared latent vector a token
// (gfx950): trees of drafts, where a sequence has hundreds to thousands of (node, head)
// rows and the products count.
//
// What bounds the kernel of few rows (latent.hpp) there is LDS: it reads a tile's keys once
// for every 16 rows.  Here a wavefront takes 32 rows, four of them 128, one wavefront a SIMD with all
// of its 512 registers, 32 tokens at a time on v_mfma_f32_32x32x16:
//   S^T [32 tokens][32 rows] = C Q^T    a wavefront: its own rows, Q (144 registers) stays with it
//   O^T [128 of 512 columns][128 rows] = C^T P^T   a wavefront: a quarter of the columns
//                                       of all rows, 256 accumulators
// A row's scores are all in one wavefront (two lanes), so that its maximum needs no exchange;
// the weights P go to the other wavefronts by LDS, in the order in which the second product
// takes them.  A tile's keys are read four times and its values once: 220 KB of LDS for
// 8.9 MFLOP, 1700 cycles beside the matrix cores' 2200.
//
// The phases overlap in one wavefront's own order: the next tile's S is multiplied while this tile's
// scores become weights (vector instructions between matrix instructions), and there is one
// barrier a tile, with the last steps of S behind it, in whose time the second product's
// first operands arrive.  Tiles come by loads that write LDS into a ring of four: one
// for the values, one for the keys, one that has arrived, one on its way.  The rotary part of a
// tile is of no use once its S is made: half of the tile's P takes its place (so d_rope is 64 here, and
// d_latent 512).
//
// What bounds it, on MI355X: the rate of matrix instructions that the card sustains.  A tile takes 1.83 to 2.1 us
// (1.25 to 1.09 PFLOP/s; the library's product of 8192^3 reaches 1.23), and no less (2.0 to 2.25) with the
// exponentials, the reads of K or V or the tile loads left out.  Beside the tiles a workgroup's Q (147 KB) and
// its O (262 KB where it is a part) cost as much as 16 tiles, which the dealing of the tiles counts (kWideFixedTiles),
// and the join of the parts of cut blocks 15 to 25 us: 8 trees of 32 nodes, 128 heads, up to 6000 tokens
// 241 + 24 us (399 + 17 with 64 rows a workgroup), 1 of 64 nodes, 16 heads, 100000 tokens 212 + 15 (282 + 10); in a long row of
// calls, on a warm card, 268 + 26 and 249 + 17.
//
// The weights P are rounded to the operands' type, half a step each, as in latent.hpp; S, maxima, sums and O are float32.
#pragma once

#include "latent.hpp"

namespace sd {
namespace latent {

// O lives in the 256 accumulation registers, block K of 32 columns by 32 rows in a[16 K .. 16 K + 15], by name: the
// compiler knows that these statements overwrite all of them and otherwise nothing of O.  (Left to
// place it, it moves O between the two halves of the registers and Q to memory.)  It has no use for
// them itself, which tests/test_wide_registers.py holds it to.  The wait states between these and
// ordinary vector instructions are their own: two before a product whose operand one may have written,
// some behind what a product takes as its third; between a product and a read of its result
// there is a whole S, or the waits at the end of the loop.
#define SD_TEN(N) "a" #N "0", "a" #N "1", "a" #N "2", "a" #N "3", "a" #N "4", "a" #N "5", "a" #N "6", "a" #N "7", "a" #N "8", "a" #N "9"
#define SD_ALL_ACCS                                                                                                  \
  SD_TEN(), SD_TEN(1), SD_TEN(2), SD_TEN(3), SD_TEN(4), SD_TEN(5), SD_TEN(6), SD_TEN(7), SD_TEN(8), SD_TEN(9),        \
      SD_TEN(10), SD_TEN(11), SD_TEN(12), SD_TEN(13), SD_TEN(14), SD_TEN(15), SD_TEN(16), SD_TEN(17), SD_TEN(18),     \
      SD_TEN(19), SD_TEN(20), SD_TEN(21), SD_TEN(22), SD_TEN(23), SD_TEN(24), "a250", "a251", "a252", "a253", "a254", \
      "a255"
template <class T, int K>
__device__ __forceinline__ void acc_mul(u32x4 a, u32x4 b) {
  if constexpr (std::is_same_v<T, Bf16>)
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 a[%2:%3], %0, %1, a[%2:%3]" ::"v"(a), "v"(b), "n"(16 * K), "n"(16 * K + 15) : SD_ALL_ACCS);
  else
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 a[%2:%3], %0, %1, a[%2:%3]" ::"v"(a), "v"(b), "n"(16 * K), "n"(16 * K + 15) : SD_ALL_ACCS);
}
template <int I>
__device__ __forceinline__ void acc_times(float f) {
  float y;
  asm volatile("v_accvgpr_read_b32 %0, a[%2]\n\tv_mul_f32 %0, %0, %1\n\tv_accvgpr_write_b32 a[%2], %0"
               : "=&v"(y)
               : "v"(f), "n"(I)
               : SD_ALL_ACCS);
}
template <int K>
__device__ __forceinline__ void acc_scale(float f) {
  each<16>([&](auto el) { acc_times<16 * K + decltype(el)::value>(f); });
  asm volatile("s_nop 7");
}
template <int K>
__device__ __forceinline__ void acc_zero(u32x4 zero) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 a[%1:%2], %0, %0, 0" ::"v"(zero), "n"(16 * K), "n"(16 * K + 15) : SD_ALL_ACCS);
}
template <int I>
__device__ __forceinline__ float acc_read() {
  float y;
  asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(y) : "n"(I));
  return y;
}
// A run of tiles starts with Q and ends with its part of O, whatever its length.  So where the list of tiles is
// dealt out, every block of rows has in front of its tiles a place as long as these take: a workgroup that comes
// into the next block gets fewer tiles.  In tiles of 64 tokens; in us (both kernels) with 0 / 4 / 8 / 12:
//   24 trees of 20 nodes, 32 heads, up to 5003: 181 / 166 / 155 / 164    8 of 32, 128 heads, up to 6000: 293 / 273 / 264 / 273
//   1 of 64, 16 heads, 100000: 240 / 222 / 227 / 233                     64 of 16, 16 heads, up to 6400: 195 / 179 / 172 / 178
// And where the longest block is no longer than a workgroup's share, and as many blocks as a workgroup gets at most take no
// longer than a share with a cut block's cost, none is cut: 8 trees of 32 nodes, 128 heads, up to 400 tokens 77 / 62,
// 30 of 46, 16 heads, up to 383 tokens 64 / 57, 48 of 64, 16 heads, 300 tokens 114 / 109 (with longer ones
// uncut too, 8 of 32, 128 heads, up to 1600 117 / 122).
// (In the kernel of few rows the first gives 1 to 9 % and takes from a chain of nodes that its sums are
// the chain form's bit by bit: not there.)
constexpr int kWideFixedTiles = 8;
// How many of a block's first `rows` rows are w, w + 4, w + 8 and so on: a wavefront's at the output.
__host__ __device__ constexpr int rows_of_wave(int rows, int w) { return rows > w ? (rows - w + 3) / 4 : 0; }
template <class T>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void latent_wide_kernel(Args a) {
  constexpr int DC = 512, C = (DC + kRope) / 8, TK = 32, kFixed = kWideFixedTiles, kRing = 4, TW = TK / 4, NL = TW * C / 64, KS = C / 2;
  constexpr int kTok = 16 * C, kBuf = TK * kTok;  // bytes of a token, of a tile
  constexpr int kAhead = 3, kFrags = 4;           // steps that K's operands are read ahead
  constexpr int kBehind = 6;                      // steps of S behind the barrier
  static_assert(NL * 64 == TW * C && KS % 4 == 0, "whole loads, steps by fours");
  __shared__ __align__(16) char ring[kRing * kBuf];
  __shared__ __align__(16) char other[2][4096];  // the half of P that is not in the tile's rotary part
  __shared__ uint64_t kin[kWideRows];            // a row's node and its ancestors
  __shared__ float fac[2][kWideRows];
  __shared__ uint32_t moved[2];  // a byte a wavefront; bit 0: its rows' references moved; 1: values that are no numbers
  __shared__ uint32_t present[kRing];             // which tokens of a tile are there
  __shared__ uint32_t offs[NL][64];               // the byte offsets of a wavefront's pieces from its first token
  __shared__ float sums[kWideRows], refs[kWideRows];
  __shared__ int uncut;  // (in LDS: it is asked once a run, and registers are short)

  const int t = threadIdx.x, lane = t & 63, n = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int L = blockIdx.x, i8 = L / 8, team = i8 / a.p.team * 8 + L % 8, member = i8 % a.p.team;

  // this team's run of the list of all sequences' tiles of 64 tokens
  auto supers_of = [&](int rows) { return (rows * a.H + kWideRows * a.p.team - 1) / (kWideRows * a.p.team); };
  auto units_of = [&](int tiles, int rows) { return (tiles + (tiles > 0 ? kFixed : 0)) * supers_of(rows); };
  auto tiles_at = [&](int b0) {
    const int bb = min(b0 + lane, a.B - 1);
    return b0 + lane < a.B ? units_of(tiles_of(length_of(a, bb)), rows_of(a, bb)) : 0;
  };
  auto scan = [&](int v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(v, d);
      if (lane >= d) v += o;
    }
    return v;
  };
  int total = 0, blocks = 0, longest = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    total += __builtin_amdgcn_readlane(scan(tiles_at(b0)), 63);
    const int bb = min(b0 + lane, a.B - 1), nt = tiles_of(length_of(a, bb));
    blocks += __builtin_amdgcn_readlane(scan(b0 + lane < a.B && nt > 0 ? supers_of(rows_of(a, bb)) : 0), 63);
    longest = max(longest, nt);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) longest = max(longest, __shfl_xor(longest, d));
  const int teams = min(a.p.teams, total);
  if (team >= teams) return;
  const int share = total / teams, more = total - share * teams;
  const int begin = team * share + min(team, more);
  int left = share + (team < more ? 1 : 0);
  // Short blocks are not cut where that takes no longer: an end that falls into a block goes to its nearer end.
  const int most = (blocks + teams - 1) / teams;
  if (t == 0) uncut = longest <= share && (int64_t)most * total <= (int64_t)blocks * (share + kFixed);
  int b = 0, within = 0;
  for (int b0 = 0, at = 0;; b0 += 64) {
    const int mine = tiles_at(b0), upto = scan(mine);
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

  auto rare = [&](int v) {  // what is computed from it is not kept in registers
    asm volatile("" : "+v"(v));
    return v;
  };
  auto piece_token = [&](int i, int ln) { return (8 * i + (ln >> 3)) / (C / 8); };
  auto piece_col = [&](int i, int ln) {
    const int tok = piece_token(i, ln), pc = 64 * i + ln - tok * C;
    return ((pc & ~7) | ((pc ^ perm(tok)) & 7)) * 8;
  };
  const bool rowed = a.token_stride < (1 << 24);
  if (w == 0)
#pragma unroll 1
    for (int i = 0; i < NL; ++i)
      offs[i][lane] = 2u * (uint32_t)(piece_token(i, lane) * (int)a.token_stride + piece_col(i, lane));
  // K: token n, piece 2 s + hf of step s; the permutation turns its low bits
  Lds krow[4];  // (in the tile that is read)
#pragma unroll
  for (int k = 0; k < 4; ++k) krow[k] = lds_of(ring) + n * kTok + (((2 * k + hf) ^ perm(n)) & 7) * 16;
  // V: lanes 4 r .. 4 r + 3 of a group of 16 read token 4 hf + r (and 8 and 16 later), 16 columns together
  int vrow[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int tok = 4 * hf + ((lane & 15) >> 2), ch = 4 * k + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    vrow[k] = tok * kTok + w * 256 + ((ch ^ perm(tok)) & 7) * 16 + 8 * (lane & 1);
  }
  // P: a lane's 16 bytes of a block of 32 rows, tokens 4 hf .. + 3 and 8 later of 16: the first 16 in the tile's
  // rotary part, the second in `other`
  const int prow = (lane >> 3) * kTok + 1024 + (lane & 7) * 16;
  const Lds tiles = lds_of(ring), weights = lds_of(other);

  __syncthreads();

  for (int seg = 0; left > 0; ++seg) {
    const int len = __builtin_amdgcn_readfirstlane(length_of(a, b)), nt = tiles_of(len);
    const int nrow = __builtin_amdgcn_readfirstlane(rows_of(a, b)), units = units_of(nt, nrow);
    if (within >= units) {
      within -= units;
      ++b;
      --seg;
      continue;
    }
    const int super = within / (nt + kFixed), u0 = within - super * (nt + kFixed), u1 = min(u0 + left, nt + kFixed);
    int t0 = max(u0 - kFixed, 0), t1 = max(u1 - kFixed, 0);
    within += u1 - u0;
    left -= u1 - u0;
    if (uniform((uint32_t)uncut)) {
      t0 = 2 * u0 >= nt + kFixed ? nt : 0;
      t1 = 2 * u1 >= nt + kFixed ? nt : 0;
    }
    if (t0 == t1) {
      --seg;
      continue;
    }
    const int slot = seg == 0 ? 0 : 1;
    const bool whole = t0 == 0 && t1 == nt;
    if (member == 0 && t == 0) {
      if (t0 == 0) a.first[(int64_t)b * a.p.supers + super] = whole ? -1 : 2 * team + slot;
      if (t1 == nt) a.last[(int64_t)b * a.p.supers + super] = team;
    }
    const int r0 = (super * a.p.team + member) * kWideRows;
    if (r0 >= nrow * a.H) continue;
    const int rlast = min(r0 + kWideRows, nrow * a.H) - 1;
    // tokens that all rows see, and that some do
    const int lim_lo = max(len - nrow, 0), lim_hi = max(len - nrow + rlast / a.H + 1, 0);
    const int from = t0 * kTile, count = (max(min(t1 * kTile, lim_hi) - from, 0) + TK - 1) / TK;  // tiles of 32

    const int32_t* table = a.pages ? a.pages + (int64_t)b * a.pages_stride : nullptr;
    // Where this wavefront's tokens of 64 tiles lie, a tile a lane: the page, if they are all in it, kNoPage if it does
    // not exist, kSlow for another kind; and their place in the page.
    constexpr int kNoPage = -1, kSlow = -2;
    int pagev = kNoPage, inv = 0;
    auto look = [&](int tl) {  // for tiles tl .. tl + 63
      const int j0 = from + (tl + lane) * TK + TW * w, pg = table ? j0 / a.page_size : 0;
      inv = table ? j0 - pg * a.page_size : j0;
      const bool plain = rowed && j0 + TW <= lim_hi && (!table || inv + TW <= a.page_size);
      const int page = plain ? (table ? load_global<int32_t>(table + pg) : b) : kSlow;
      pagev = !plain || (page >= 0 && page < a.n_pages) ? page : kNoPage;
    };
    // What a tile's loads need where they go by a view, one after another: on says that they do.  In parts, for the
    // time of matrix instructions.
    struct Load {
      uint32_t lo, hi;
      int64_t at;
      int page, in;
    } ld;
    const int64_t span = 2 * ((TW - 1) * a.token_stride + DC + kRope);
    auto ask = [&](int tl) {
      ld.page = __builtin_amdgcn_readlane(pagev, tl & 63);
      ld.in = __builtin_amdgcn_readlane(inv, tl & 63);
    };
    auto place = [&] { ld.at = (int64_t)max(ld.page, 0) * a.page_stride; };
    auto point = [&] {
      const uint64_t to = reinterpret_cast<uint64_t>(a.cache + ld.at + (int64_t)ld.in * (int)a.token_stride);
      ld.lo = uniform((uint32_t)to);
      ld.hi = uniform((uint32_t)(to >> 32));
    };
    // The same for a tile of another kind, token by token.
    auto load_slow = [&](int tl) {
      const int j0 = from + tl * TK + TW * w;
      const Lds dst = tiles + (tl & 3) * kBuf + TW * w * kTok;
      const int have = min(max(lim_hi - j0, 0), TW), ln = rare(lane), j = j0 + ln % TW, pg = table ? j / a.page_size : 0;
      const int page = ln % TW < have ? (table ? load_global<int32_t>(table + pg) : b) : -1;
      const bool ok = page >= 0 && page < a.n_pages;
      const uint32_t valid = (uint32_t)__ballot(ok) & ((1u << TW) - 1u);
      const uint64_t adr = reinterpret_cast<uint64_t>(
          a.cache + (ok ? (int64_t)page * a.page_stride + (int64_t)(table ? j - pg * a.page_size : j) * a.token_stride : 0));
#pragma unroll 1
      for (int i = 0; i < NL; ++i) {
        const int tok = piece_token(i, ln), col = piece_col(i, ln);
        const uint32_t lo = __shfl((int)(uint32_t)adr, tok), hi = __shfl((int)(uint32_t)(adr >> 32), tok);
        if (valid >> tok & 1u) load_lds((Global)(((uint64_t)hi << 32) | lo) + 2 * col, dst + 1024 * i);
      }
      return valid;
    };
    auto load_piece = [&](auto i, int tl, uint32_t off, uint32_t on) {
      load_lds_view<1024 * decltype(i)::value>(u32x4{ld.lo, ld.hi, (uint32_t)span, kBufferWord3}, off,
                                               lds_address(tiles + (tl & 3) * kBuf + TW * w * kTok),
                                               (uint64_t)0 - (uint64_t)(on & 1u));
    };
    // a tile's loads have arrived: zeros for tokens that no row sees, or of no page
    auto arrived = [&](int tl, uint32_t valid) {
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
      if (valid != (1u << TW) - 1u) {
        const Lds dst = tiles + (tl & 3) * kBuf + TW * w * kTok;
        for (int i = rare(lane); i < TW * C; i += 64)
          if (!(valid >> (i / C) & 1u)) *(__attribute__((address_space(3))) u32x4*)(dst + 16 * i) = u32x4{0u, 0u, 0u, 0u};
        __builtin_amdgcn_s_waitcnt(0);
      }
    };
    auto note = [&](int tl, uint32_t valid) {
      if (lane == 0) reinterpret_cast<uint8_t*>(&present[tl & 3])[w] = (uint8_t)valid;
    };

    // the first tiles on their way, then this wavefront's rows of Q
    uint32_t held = 0;  // a byte a tile: the tokens that it brings
    look(0);
#pragma unroll 1
    for (int k = 0; k < min(count, 3); ++k) {
      ask(k);
      place();
      point();
      const uint32_t on = uniform(~(uint32_t)ld.page >> 31);
      each<NL>([&](auto i) { load_piece(i, k, offs[decltype(i)::value][lane], on); });
      held |= (ld.page >= 0 ? (1u << TW) - 1u : ld.page == kNoPage ? 0u : uniform(load_slow(k))) << (8 * k);
    }
    int up = -1;
    if (w == 0 && lane < nrow) up = load_global<int32_t>(a.parents + (int64_t)b * a.Q + lane);
    u32x4 qf[KS];
    {
      const int row = min(r0 + 32 * w + n, rlast), i = row / a.H, h = row - i * a.H;
      const uint16_t* src = a.q + (int64_t)b * a.qs + (int64_t)i * a.qr + (int64_t)h * a.qh + 8 * hf;
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = load_global<u32x4>(src + 16 * k) ^ a.flip;
    }
    if (w == 0) {
      const uint64_t set = ancestors(up < lane ? up : -1, lane);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = min(r0 + 64 * k + lane, rlast);
        kin[64 * k + lane] = (uint64_t)__shfl((unsigned long long)set, row / a.H);
      }
    }
    float m = -INFINITY, l = 0.f;
    bool marked = false;
    u32x4 kf[kFrags];
    // Step s takes columns 16 at(s) ..: the rotary part first, so that it has been read before the barrier
    // behind which its place is taken.
    auto at = [](int s) { return s < 4 ? s + KS - 4 : s - 4; };
    auto kread = [&](int s) { kf[s % kFrags] = lds_read<u32x4>(krow[s & 3] + (at(s) >> 2) * 128); };
    auto kmove = [&](int tl) {  // to tile tl from the one before
      const int by = (tl & 3) == 0 ? -3 * kBuf : kBuf;
#pragma unroll
      for (int k = 0; k < 4; ++k) krow[k] += by;
    };
    __builtin_amdgcn_s_waitcnt(0);
#pragma unroll 1
    for (int k = 0; k < min(count, 2); ++k) {
      arrived(k, held >> (8 * k) & 0xffu);
      note(k, held >> (8 * k) & 0xffu);
    }
    __syncthreads();
    // S of the first tile
    f32x16 sa, sb;
#pragma unroll
    for (int i = 0; i < 16; ++i) sa[i] = 0.f;
    if (count > 0) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) kread(s);
      each<KS>([&](auto step) {
        constexpr int s = decltype(step)::value;
        if constexpr (s + kAhead < KS) kread(s + kAhead);
        sa = T::mfma32(kf[s % kFrags], qf[at(s)], sa);
      });
    }
    uint32_t seen = count > 0 ? uniform(present[0]) : 0u, valid = held >> 16;
    kmove(1);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) kread(s);
    const u32x4 zero{0u, 0u, 0u, 0u};
    each<16>([&](auto blk) { acc_zero<decltype(blk)::value>(zero); });
    // the first tile's weights take the place of its rotary parts, which all wavefronts have read now
    lds_barrier();
    // wait states for a read of the last results behind a branch
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7");
    __builtin_amdgcn_sched_barrier(0);

    // One tile, whose scores are in sc; the next one's go to nx.  EDGE: of tokens that some rows do not see.
    auto tile = [&](auto kind, int tl, f32x16& sc, f32x16& nx) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(kind)::value;
      const Lds here = tiles + (tl & 3) * kBuf;
      const int first = from + tl * TK;
      uint32_t flags = 0;
      if (EDGE || seen != ~0u) {
        const int ln = rare(lane);
        uint32_t sees = ~0u;
        if constexpr (EDGE) {
          const int node = first - (len - nrow);  // the node of the tile's first token
          const uint64_t set = kin[32 * w + (ln & 31)];
          sees = node >= 64   ? 0u
                 : node >= 0  ? (uint32_t)(set >> node)
                 : node > -32 ? ((uint32_t)set << -node) | ((1u << -node) - 1u)
                              : ~0u;
        }
        sees = (sees & seen) >> (4 * (ln >> 5));
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = sees & (1u << (8 * (i >> 2) + (i & 3))) ? sc[i] : -INFINITY;
        // A token that some rows see and others do not: their weight for it is 0, and 0
        // times an infinity or NaN is not.
        if constexpr (EDGE) {
          uint32_t bad = 0;
          const int lo = max(lim_lo - first, 0), hi = min(lim_hi - first, TK);
          for (int i = rare(t); i < (hi - lo) * DC / 2; i += 256)
            bad |= lawless<T>(lds_read<uint32_t>(here + (lo + i / (DC / 2)) * kTok + (i % (DC / 2)) * 4));
          flags = __any((bad & 0x80008000u) != 0) ? 2u : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) nx[i] = 0.f;
      // S of the next tile, and between its steps this tile's weights
      float mx = 0.f, ref = 0.f, p[16];
      auto soften = [&](auto step) {
        constexpr int s = decltype(step)::value;
        if constexpr (s == 0) mx = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(sc[4], sc[5]));
        if constexpr (s == 1) mx = fmaxf(mx, fmaxf(fmaxf(sc[6], sc[7]), fmaxf(fmaxf(sc[8], sc[9]), sc[10])));
        if constexpr (s == 2) mx = fmaxf(mx, fmaxf(fmaxf(sc[11], sc[12]), fmaxf(fmaxf(sc[13], sc[14]), sc[15])));
        if constexpr (s == 3) mx = across(mx, true, true) * a.c;
        if constexpr (s == 4) {
          if (const bool over = mx > reach<T>(m); __any(over)) {
            if (__any(over && m != -INFINITY)) flags |= 1u;  // (O is 0 where there was no reference yet)
            const float to = over ? reference<T>(mx) : m, f = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
            if (hf == 0) fac[tl & 1][32 * w + n] = f;
          }
          if (lane == 0) reinterpret_cast<uint8_t*>(&moved[tl & 1])[w] = (uint8_t)flags;
          ref = m == -INFINITY ? 0.f : m;
        }
        if constexpr (s >= 5 && s < 21) {
          constexpr int i = s - 5;
          p[i] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[i], a.c, -ref));
          l += p[i];
        }
        if constexpr (s == 14)
          *(__attribute__((address_space(3))) u32x4*)(here + prow + w * 8 * kTok) =
              u32x4{T::pack(p[0], p[1]), T::pack(p[2], p[3]), T::pack(p[4], p[5]), T::pack(p[6], p[7])};
        if constexpr (s == 23) {
          if (((tl + 3) & 63) == 0) look(tl + 3);
          ask(tl + 3);
        }
        if constexpr (s == 24) place();
        if constexpr (s == 26) point();
        if constexpr (s == 22)
          *(__attribute__((address_space(3))) u32x4*)(weights + (tl & 1) * 4096 + w * 1024 + lane * 16) =
              u32x4{T::pack(p[8], p[9]), T::pack(p[10], p[11]), T::pack(p[12], p[13]), T::pack(p[14], p[15])};
      };
      each<KS - kBehind>([&](auto step) {
        constexpr int s = decltype(step)::value;
        if constexpr (s + kAhead < KS) kread(s + kAhead);
        __builtin_amdgcn_sched_barrier(0);
        nx = T::mfma32(kf[s % kFrags], qf[at(s)], nx);
        soften(step);
        __builtin_amdgcn_sched_barrier(0);
      });
      if (tl + 2 < count) arrived(tl + 2, valid);
      lds_barrier();
      u32x4 pf[6], vf[2];  // P's block r: place r, of the second 16 tokens 4, 5, 0 and 1
      auto vread = [&](int i) {  // block i % 4 of 32 columns, tokens 16 (i / 4) ..
        const Lds src = here + vrow[i & 1] + (i >> 1 & 1) * 128 + 16 * (i >> 2) * kTok;
        const u32x2 lo = lds_read_tr(src), hi = lds_read_tr(src + 8 * kTok);
        vf[i & 1] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      };
      uint32_t said = moved[tl & 1];
#pragma unroll
      for (int r = 0; r < 4; ++r) pf[r] = lds_read<u32x4>(here + prow + r * 8 * kTok);
      auto second = [&](int r) { pf[(r + 4) % 6] = lds_read<u32x4>(weights + (tl & 1) * 4096 + r * 1024 + lane * 16); };
      vread(0);
      seen = present[(tl + 1) & 3];
      uint32_t go = offs[0][lane];
      each<kBehind>([&](auto step) {
        constexpr int s = KS - kBehind + decltype(step)::value;
        if constexpr (s + kAhead < KS) kread(s + kAhead);
        __builtin_amdgcn_sched_barrier(0);
        nx = T::mfma32(kf[s % kFrags], qf[at(s)], nx);
        __builtin_amdgcn_sched_barrier(0);
      });
      if (tl + 2 < count) note(tl + 2, valid);
      const uint32_t on = uniform((~(uint32_t)ld.page & (uint32_t)(tl + 3 - count)) >> 31);
      valid = on ? (1u << TW) - 1u : 0u;
      if (tl + 3 < count && ld.page == kSlow) valid = uniform(load_slow(tl + 3));
      seen = uniform(seen);
      said = uniform(said);
      if (said) {
        each<4>([&](auto rows) {
          constexpr int r = decltype(rows)::value;
          if (said >> (8 * r) & 1u) {
            const float f = fac[tl & 1][32 * r + n];
            acc_scale<r>(f);  // block 4 c + r: columns 32 c .. of the wavefront's, rows 32 r ..
            acc_scale<4 + r>(f);
            acc_scale<8 + r>(f);
            acc_scale<12 + r>(f);
          }
        });
        if (EDGE && (said & 0x02020202u)) {
          // What the infinities and NaN give to the rows that see them goes to this segment's place in the
          // workspace (each lane to the elements of O that it holds), and zeros to their own places.
          const int ln = rare(lane), lo = max(lim_lo - first, 0), hi = min(lim_hi - first, TK);
          float* mine = a.part + (((int64_t)L * 2 + slot) * kWideRows + (ln & 31)) * DC + w * 128 + 4 * (ln >> 5);
          if (!marked) {
#pragma clang loop unroll(disable)
            for (int k = 0; k < 64; ++k) *reinterpret_cast<f32x4*>(mine + (k >> 4) * 32 * DC + 8 * (k & 15)) = f32x4{0.f, 0.f, 0.f, 0.f};
            marked = true;
          }
#pragma clang loop unroll(disable)
          for (int j = lo; j < hi; ++j) {
            const int at = (ln & 31) + 32 * (j >> 2 & 1), part = 4 * (j >> 3 & 1) + (j & 3);
#pragma clang loop unroll(disable)
            for (int k = 0; k < 16; ++k) {  // four columns
              const int ch = w * 16 + k, pc = (ch & ~7) | ((ch ^ perm(j)) & 7);
              const u32x2 v = lds_read<u32x2>(here + j * kTok + pc * 16 + 8 * (ln >> 5));
              if (!((lawless<T>(v[0]) | lawless<T>(v[1])) & 0x80008000u)) continue;
#pragma clang loop unroll(disable)
              for (int r = 0; r < 4; ++r) {
                if (!(kin[32 * r + (ln & 31)] >> (first + j - (len - nrow)) & 1u)) continue;
                const Lds src = j < 16 ? here + (8 * r + (at >> 3)) * kTok + 1024 + (at & 7) * 16
                                       : weights + (tl & 1) * 4096 + r * 1024 + at * 16;
                const float p = T::value(lds_read<uint16_t>(src + 2 * part));
                float* to = mine + r * 32 * DC + 8 * k;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint16_t x = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
                  if ((x & T::kExponent) == T::kExponent) to[i] += p * T::value(x);
                }
              }
            }
          }
          __syncthreads();
          for (int i = rare(t); i < hi * DC; i += 256) {
            const Lds v = here + (i / DC) * kTok + 2 * (i % DC);
            if (i / DC >= lo && (lds_read<uint16_t>(v) & T::kExponent) == T::kExponent)
              *(__attribute__((address_space(3))) uint16_t*)v = 0;
          }
          __syncthreads();
          vread(0);
        }
      }
      // O^T += C^T P^T; the next tile's loads go out between the products, and the first keys of the one
      // behind it are read at their end
      each<8>([&](auto step) {
        constexpr int i = decltype(step)::value;
        if constexpr (i == 2) {
          second(0);
          second(1);
        }
        if constexpr (i + 1 < 8) vread(i + 1);
        if constexpr (i == 7) {
          kmove(tl + 2);
#pragma unroll
          for (int s = 0; s < kAhead; ++s) kread(s);
        }
        __builtin_amdgcn_sched_barrier(0);
        load_piece(step, tl + 3, go, on);
        go = offs[i + 1][lane];
        if constexpr (i == 7) load_piece(std::integral_constant<int, 8>{}, tl + 3, go, on);
        each<4>([&](auto rows) {
          constexpr int r = decltype(rows)::value, k = 4 * (i & 3) + r;
          acc_mul<T, k>(vf[i & 1], pf[i < 4 ? r : (r + 4) % 6]);
          if constexpr (i == 3 && r < 2) second(r + 2);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    const int whole_tiles = min(max(lim_lo - from, 0) / TK, count);  // that all rows see
    // (two in turn, so that no scores are moved; an odd one and the few that some rows do not see take theirs along)
    int tl = 0;
#pragma unroll 1
    for (; tl + 1 < whole_tiles; tl += 2) {
      tile(std::false_type{}, tl, sa, sb);
      tile(std::false_type{}, tl + 1, sb, sa);
    }
#pragma unroll 1
    for (; tl < count; ++tl) {
      tile(std::true_type{}, tl, sa, sb);
      sa = sb;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) krow[k] -= ((count + 1) & 3) * kBuf;
    // wait states for a read of the last results behind the loop's branch
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7");
    __builtin_amdgcn_sched_barrier(0);

    l = across(l, true, false);
    if (hf == 0) {
      sums[32 * w + n] = l;
      refs[32 * w + n] = m;
    }
    __syncthreads();
    // Rows w + 4 j, j = 0 .. 31, leave by this wavefront; lane j knows where to, and the row's 1 / sum.
    const int own = w + 4 * n, row = r0 + own;
    const float sum = sums[own], ref = refs[own];
    uint64_t to = 0;
    float f = 0.f;
    if (!whole) {
      const int64_t at = ((int64_t)L * 2 + slot) * kWideRows + own;
      to = reinterpret_cast<uint64_t>(a.part + at * DC);
      if (hf == 0) a.stat[at] = make_float2(ref, sum);
    } else if (row <= rlast) {
      const int i = row / a.H, h = row - i * a.H;
      f = sum > 0.f ? 1.f / sum : sum != sum ? NAN : 0.f;
      to = reinterpret_cast<uint64_t>(a.out + (int64_t)b * a.os + (int64_t)i * a.orow + (int64_t)h * a.oh);
      if (hf == 0 && a.lse) a.lse[((int64_t)b * a.Q + i) * a.H + h] = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    const int rows_here = whole ? rows_of_wave(rlast - r0 + 1, w) : kWideRows / 4;
    // O goes by way of the ring, in whole lines: half of the columns at a time, [128 rows][256] in pieces of 16 bytes
    // that are permuted by the row; piece 16 w + p is columns 128 w + 64 half + 4 p ..
    each<2>([&](auto which) {
      constexpr int half = decltype(which)::value;
      if (half == 1) __syncthreads();
      each<8>([&](auto blk) {
        constexpr int c = 2 * half + (decltype(blk)::value >> 2), r = decltype(blk)::value & 3, k = 4 * c + r;
        each<4>([&](auto quad) {
          constexpr int q = decltype(quad)::value, at = 16 * k + 4 * q;
          const int piece = 16 * w + 8 * (c & 1) + 2 * q + hf;
          *(__attribute__((address_space(3))) f32x4*)(tiles + (32 * r + n) * 1024 + (piece ^ n) * 16) =
              f32x4{acc_read<at>(), acc_read<at + 1>(), acc_read<at + 2>(), acc_read<at + 3>()};
        });
      });
      __syncthreads();
      const int col = (lane >> 4) * 128 + 64 * half + (lane & 15) * 4;
      const float* marks = a.part + (((int64_t)L * 2 + slot) * kWideRows + w) * DC + col;
#pragma unroll 1
      for (int j0 = 0; j0 < rows_here; j0 += 4) {
        f32x4 x[4];
        int js[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          js[k] = min(j0 + k, rows_here - 1);  // (the last row again where there are no four)
          const int at = w + 4 * js[k];
          x[k] = lds_read<f32x4>(tiles + at * 1024 + (lane ^ (at & 31)) * 16);
          if (marked) x[k] += *reinterpret_cast<const f32x4*>(marks + (int64_t)js[k] * 4 * DC);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint64_t base = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(to >> 32), js[k]) << 32) |
                                (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)to, js[k]);
          if (whole) {
            const float fj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), js[k]));
            *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(base) + col) =
                u32x2{T::pack(x[k][0] * fj, x[k][1] * fj), T::pack(x[k][2] * fj, x[k][3] * fj)};
          } else {
            *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(base) + col) = x[k];
          }
        }
      }
    });
    __syncthreads();
  }
}

template <class T>
hipError_t run_wide(const Args& a, hipStream_t s) {
  const hipError_t e = launch_timed("latent_wide", latent_wide_kernel<T>, dim3(kGroups), dim3(256), s, a);
  return e != hipSuccess ? e : join<T, 512>(a, s);
}

}  // namespace latent
}  // namespace sd
