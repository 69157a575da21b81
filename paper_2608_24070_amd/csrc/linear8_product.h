// linear8_product.h - the kernels of the 8-bit product as bodies, each of which hands its fp32 results to what it is given to
// end them with, and the plan of a product: for slim_linear8 (linear8.hip) and the products that end in an activation
// (linear8_act.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <algorithm>
#include <type_traits>

#include "slim_launch.h"
#include "slim_q8.h"
#include "slim_timing.h"

namespace {

SLIM_DEV f4_t mfma8(i32x8_t a, i32x8_t b, f4_t c, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

SLIM_DEV i32x8_t cat8(u32x4_t lo, u32x4_t hi) {
  return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// f(integral_constant 0) .. f(integral_constant N - 1)
template <int N, int I = 0, class F>
SLIM_DEV void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, I + 1>(f);
  }
}

// Four consecutive columns of one row of Y, of which `n` exist.
template <int DT>
SLIM_DEV void store4_16(uint16_t* y, int64_t at, int64_t n, f4_t v) {
  if (n >= 4) {
    const u32x2_t p = {to_16<DT>(v[0]) | to_16<DT>(v[1]) << 16, to_16<DT>(v[2]) | to_16<DT>(v[3]) << 16};
    __builtin_memcpy(y + at, &p, 8);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) y[at + e] = (uint16_t)to_16<DT>(v[e]);
  }
}

// Results as they are, in 16 bits.
template <int DT>
struct StoreRows {
  static constexpr bool kRows = false;
  static constexpr int kType = DT;
  uint16_t* Y;
  int64_t ldy;
  SLIM_DEV void four(int64_t m, int64_t n, int64_t left, f4_t v) const { store4_16<DT>(Y, m * ldy + n, left, v); }
};

// ------------------------------------------------------------------------------------- few rows
// One piece of 16 values of X in 8 bits, as k_quant8 (eight lanes share a group): used where X is quantised in the product's
// own launch.
template <int DT>
SLIM_DEV void quant16(const void* X, int64_t at, int64_t left, u32x4_t& c, uint32_t& b) {
  float f[16];
  load8<DT>(X, at, left, f);
  load8<DT>(X, at + 8, left - 8, f + 8);
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) m = max(m, q8_abs(f[e]));
  b = q8_exponent(oct_max_u32(m));
  const float s = q8_inverse(b);
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = q8_codes4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3], s);
}

// NT tiles of 16 weight rows and up to 16 FM rows of X per block; its eight waves take the groups of the reduction in turn
// and add their sums through LDS in wave order. Nothing is shared within the reduction, so weight tiles (2 KiB of
// consecutive bytes) and X fragments go straight from memory to registers, U groups of a wave in flight at once. Bound by
// the weight's bytes, and for more than a few rows by those of X, which every block reads: two tiles a block halve them.
// 28672 x 8192, M 1: 42.8 us (5.5 TB/s) for a launch by itself, operands from memory; 4096 x 4096, M 1 10.0 us, of which a launch
// is half (7.0 as one of many in a graph).
// Results go to fin.four(row, column, columns that exist, four sums).
// XT: the type of X. 3 (codes): rows are read as they are. Otherwise every block first turns the whole of X into codes in
// LDS, while its first weight tiles are on their way: worth it for the few rows whose codes fit kFewLds.
constexpr int kFewLds = 32768;
template <int FM, int NT, int U, int XT, class Fin>
SLIM_DEV void few_body(const uint8_t* __restrict__ X, const uint8_t* __restrict__ ex, int64_t ldx, int K,
                       const uint8_t* __restrict__ W, const uint8_t* __restrict__ ew, int M, int64_t N, int G, const Fin& fin) {
  constexpr bool kCodes = XT == SLIM_Q8_E4M3;
  __shared__ f4_t part[8][FM * NT][64];
  __shared__ __attribute__((aligned(16))) uint8_t xs[kCodes ? 16 : kFewLds + kFewLds / 128];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4, Ge = (G + 3) & ~3;
  const int64_t t0 = (int64_t)blockIdx.x * NT, Nt = (N + 15) / 16;
  const uint8_t* w[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) w[n] = W + (t0 + n < Nt ? t0 + n : Nt - 1) * G * 2048 + lane * 16;   // past the end: not stored
  const uint8_t* sw = ew + (t0 / 8) * Ge;                  // NT divides 8: one block of exponents
  u32x4_t wv[U][NT][2];
  auto load_w = [&](int g) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + 8 * u < G)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) wv[u][n][h] = *reinterpret_cast<const u32x4_t*>(w[n] + (int64_t)(g + 8 * u) * 2048 + 1024 * h);
  };
  load_w(wave);
  const uint8_t* xp[FM];
  const uint8_t* sx[FM];
  if constexpr (!kCodes) {
    uint8_t* es = xs + kFewLds;
    for (int i = threadIdx.x; i < M * G * 8; i += 512) {
      const int row = i / (G * 8), p = i - row * (G * 8), col = 16 * p;
      u32x4_t c;
      uint32_t b;
      quant16<XT>(X, (int64_t)row * ldx + col, (int64_t)K - col, c, b);
      *reinterpret_cast<u32x4_t*>(xs + row * G * 128 + col) = c;
      if ((p & 7) == 0) es[row * G + (p >> 3)] = (uint8_t)b;
    }
    __syncthreads();
  }
#pragma unroll
  for (int f = 0; f < FM; ++f) {
    const int m = 16 * f + r < M ? 16 * f + r : M - 1;       // rows past the last repeat it; not stored
    if constexpr (kCodes) {
      xp[f] = X + (int64_t)m * G * 128 + 32 * q;
      sx[f] = ex + (int64_t)m * Ge;
    } else {
      xp[f] = xs + m * G * 128 + 32 * q;
      sx[f] = xs + kFewLds + m * G;
    }
  }
  f4_t acc[FM][NT];
#pragma unroll
  for (int f = 0; f < FM; ++f)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[f][n] = f4_t{0.f, 0.f, 0.f, 0.f};
  for (int g = wave; g < G; g += 8 * U) {
    if (g != wave) load_w(g);
    u32x4_t xv[U][FM][2];
    int e[U][FM], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + 8 * u < G) {
        s[u] = sw[g + 8 * u];
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          xv[u][f][0] = *reinterpret_cast<const u32x4_t*>(xp[f] + (g + 8 * u) * 128);
          xv[u][f][1] = *reinterpret_cast<const u32x4_t*>(xp[f] + (g + 8 * u) * 128 + 16);
          e[u][f] = sx[f][g + 8 * u];
        }
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + 8 * u < G)
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            acc[f][n] = mfma8(cat8(wv[u][n][0], wv[u][n][1]), cat8(xv[u][f][0], xv[u][f][1]), acc[f][n], s[u], e[u][f]);
  }
#pragma unroll
  for (int f = 0; f < FM; ++f)
#pragma unroll
    for (int n = 0; n < NT; ++n) part[wave][f * NT + n][lane] = acc[f][n];
  __syncthreads();
  for (int i = wave; i < FM * NT; i += 8) {
    f4_t v = part[0][i][lane];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += part[k][i][lane];
    const int m = 16 * (i / NT) + r;
    const int64_t n = 16 * (t0 + i % NT) + 4 * q;
    if (m < M && n < N) fin.four(m, n, N - n, v);
  }
}

// ------------------------------------------------------------------------------------- many rows
// c += a b with the scale bytes J of sa and sb, written out so that the sum stays where it is: the compiler gives the
// instruction's result registers of their own and moves 256 sums around a loop that has no others free (a fifth of the
// time). The operands come from loads that were waited for and the sum was last written 15 and more products ago, so no
// wait states are needed before it.
template <int J>
SLIM_DEV void mfma8_in_place(f4_t& c, i32x8_t a, i32x8_t b, uint32_t sa, uint32_t sb) {
#if defined(__HIP_DEVICE_COMPILE__)   // the host compiler knows no accumulation registers
#define SLIM_MFMA8(sel) \
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 " sel : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb))
  if constexpr (J == 0) SLIM_MFMA8("op_sel_hi:[0,0,0]");
  if constexpr (J == 1) SLIM_MFMA8("op_sel:[1,1,0] op_sel_hi:[0,0,0]");
  if constexpr (J == 2) SLIM_MFMA8("op_sel_hi:[1,1,0]");
  if constexpr (J == 3) SLIM_MFMA8("op_sel:[1,1,0] op_sel_hi:[1,1,0]");
#undef SLIM_MFMA8
#endif
}

// What the 16-byte slots of LDS rows of 128 bytes are XORed by. A read of 16 bytes a lane takes lanes 0-3, 12-15 and 20-27 in
// one cycle, 4-11, 16-19 and 28-31 in another, and lanes 32 on alike: with this every such sixteen falls in distinct banks
// (conflicts are counted as 3 % of the LDS cycles; by the whole row they were half).
SLIM_DEV int swizzle8(int row) { return ((row >> 1) & 7) ^ (((row >> 2) ^ (row >> 3)) & 1) * 2; }

// Tiles of 16 FM rows of X by 64 WN columns, four waves of 16 FM x 64 each: WN side by side, and as many of those as are
// left over 4 / WN parts of the reduction, whose sums are added in part order at the end. A wave's weight tiles are its own:
// they go from memory to registers in whole tiles, three groups ahead. X is shared by the WN waves: per group a [16 FM][128]
// slab goes to LDS by direct loads (16 bytes a lane), three groups ahead in a ring of four. Exponents of X go the same way, one
// 32-bit word (four groups) a row; the unit picks the group's byte by itself. Fragments of X are read three ahead of their
// four MFMAs. LDS reads are written out with counted waits (the compiler cannot tell the ring's slots apart and would wait for
// every load in flight). Rows and weight tiles past the ends repeat the last one; their results are not stored.
// 256 x 256 tiles are bound by the matrix unit and by the power it draws: 8192 x 28672 x 8192 1.31 to 1.36 ms by card, 2.8 to
// 2.9 PFLOP/s (a library product of unscaled fp8 2.66): it is busy for 78 % of the cycles (8192 x 8192 x 8192) at the 1.6 GHz that the card then keeps,
// LDS for 22 %. Shorter tiles and parts of the reduction are for fewer rows, where the weight's bytes come to count: 512 x
// 28672 x 8192 98 us (2.5 PFLOP/s), 64 x 28672 x 8192 53 us (4.4 TB/s of weights), 16 x 28672 x 8192 48 us, 45 x 13824 x 5120 22 us
// (weights from memory; a launch of k_quant8 before it, 4 us), 2048 x 4096 x 4096 34 us (2.0).
// `end()` gives what the results go to; it is asked for after the loop, whose registers are all taken.
template <int FM, int WN, class End>
SLIM_DEV void tile_body(const uint8_t* __restrict__ X, const uint8_t* __restrict__ ex, const uint8_t* __restrict__ W,
                        const uint8_t* __restrict__ ew, int64_t M, int64_t N, int G, int fours, float* __restrict__ sums, const End& end) {
#if defined(__HIP_DEVICE_COMPILE__)   // the host compiler takes no part in the written-out instructions below
  constexpr int TM = 16 * FM, TN = 64 * WN, WK = 4 / WN;     // rows and columns of a tile; parts of the reduction
  // a group's barrier stands before fragment FB, since the next slab's fragments are read three ahead; a wave's P direct
  // loads of a slab follow from there, kXper at a fragment, the eight of a weight tile start at fragment 0, kWper at one
  constexpr int P = TM / (8 * WN), FB = FM < 6 ? FM - 3 : FM / 2;
  constexpr int kXper = (P + FM - FB - 1) / (FM - FB), kWper = FM < 8 ? 8 / FM : 1;
  constexpr uint32_t kSlab = TM * 128, kE = 4 * kSlab, kPart = kE + 2 * TM * 4;
  static_assert(FM % 4 == 0 && WK * kPart >= (WK > 1 ? 4 * FM * 4096 : 4 * TM * 128));
  __shared__ __attribute__((aligned(16))) uint8_t lds[WK * kPart];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4, wi = wave % WN, part = wave / WN;
  // block b runs on XCD b % 8, which takes positions [x Q, (x + 1) Q) of an order that walks bands of about 1024 rows column
  // by column: the blocks that run together on one XCD share slabs of X and weight tiles in its L2
  constexpr uint32_t kBand = 1024 / TM;
  const uint32_t tn = (uint32_t)((N + TN - 1) / TN), tm = (uint32_t)((M + TM - 1) / TM), T = tn * tm, Q = (T + 7) / 8;
  const uint32_t pos = (blockIdx.x % 8) * Q + blockIdx.x / 8;
  if (pos >= T) return;
  const uint32_t band = pos / (kBand * tn), q0 = pos - band * kBand * tn;
  const uint32_t width = tm - band * kBand < kBand ? tm - band * kBand : kBand, nt = q0 / width;
  // (divisions run on the vector unit: back to scalars)
  const int64_t m0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(band * kBand + q0 - nt * width)) * TM;
  const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane((int)nt) * TN;
  const int Ge = (G + 3) & ~3;
  const int64_t Nt = (N + 15) / 16;
  const int rows = (int)(M - m0 < TM ? M - m0 : TM), wt = (int)(Nt - n0 / 16 < 4 * WN ? Nt - n0 / 16 : 4 * WN);
  const rsrc_t rx = make_rsrc(X + m0 * G * 128, (int64_t)rows * G * 128), re = make_rsrc(ex + m0 * Ge, (int64_t)rows * Ge);
  const rsrc_t rw = make_rsrc(W + (n0 / 16) * G * 2048, (int64_t)wt * G * 2048);
  const int64_t nb = (n0 + 64 * wi) / 128, nbs = (N + 127) / 128;
  const uint32_t* sew = reinterpret_cast<const uint32_t*>(ew + (nb < nbs ? nb : nbs - 1) * Ge);

  // lane L of a direct load writes LDS bytes 16 L of eight rows: row L / 8, physical slot L % 8
  uint32_t xo[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int row = wi * (TM / WN) + 8 * p + (lane >> 3);
    xo[p] = (uint32_t)(row < rows ? row : rows - 1) * (uint32_t)(G * 128) + (uint32_t)(((lane & 7) ^ swizzle8(row)) * 16);
  }
  const int ew0 = (wi % (TM / 64)) * 64;
  const uint32_t eo = (uint32_t)(ew0 + lane < rows ? ew0 + lane : rows - 1) * (uint32_t)Ge;
  uint32_t wo[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) wo[f] = (uint32_t)(4 * wi + f < wt ? 4 * wi + f : wt - 1) * (uint32_t)(G * 2048);
  const uint32_t wl = (uint32_t)lane * 16u;
  uint8_t* const ring = lds + (uint32_t)part * kPart;
  auto issue_x = [&](int c, auto zc, auto pc) {                 // piece p of this wave's part of a slab
    const uint32_t cc = (uint32_t)(c < G ? c : G - 1);          // past the end: a dead slot
    constexpr int p = decltype(pc)::value;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_ptr_t)&ring[decltype(zc)::value * kSlab + (uint32_t)(wi * (TM / WN) + 8 * p) * 128u],
                                             16, xo[p], cc * 128u, 0, 0);
  };
  auto issue_e = [&](int w) {                               // word w of the rows' exponents
    const uint32_t ww = (uint32_t)(w < Ge / 4 ? w : Ge / 4 - 1);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(re, (lds_ptr_t)&ring[kE + (uint32_t)(w & 1) * (TM * 4) + (uint32_t)ew0 * 4u], 4, eo, ww * 4u, 0, 0);
  };
  struct Wt { u32x4_t v[4][2]; };
  auto load_w = [&](Wt& w, int c, auto ic) {                    // half i % 2 of tile i / 2 of group c, zeros past the last
    constexpr int f = decltype(ic)::value >> 1, h = decltype(ic)::value & 1;
    const uint32_t at = c < G ? wl : 0x80000000u;               // past the resource: zeros, no memory access
    w.v[f][h] = __builtin_amdgcn_raw_buffer_load_b128(rw, at + 1024u * h, wo[f] + (uint32_t)(c < G ? c : 0) * 2048u, 0);
  };

  f4_t acc[FM][4];
#pragma unroll
  for (int f = 0; f < FM; ++f)
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[f][n] = f4_t{0.f, 0.f, 0.f, 0.f};

  // fragment f of a slab: rows 16 f + r, codes 32 q .. + 31 in two 16-byte slots; slabs 2 and 3 have bases of their own,
  // so that every offset fits the 16-bit immediate
  struct Frag { u32x4_t h[2]; };
  const uint32_t lb = (uint32_t)(uintptr_t)(lds_ptr_t)&ring[0];
  uint32_t xa[2][2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    xa[0][h] = lb + (uint32_t)(r * 128 + (((2 * q + h) ^ swizzle8(r)) * 16));
    xa[1][h] = xa[0][h] + 2 * kSlab;
  }
  auto rd = [&](Frag& F, auto zc, auto fc) {
    constexpr int z = decltype(zc)::value, f = decltype(fc)::value;
    constexpr uint32_t off = (z & 1) * kSlab + f * 2048;
    const uint32_t a0 = xa[z >> 1][0], a1 = xa[z >> 1][1];
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(F.h[0]) : "v"(a0), "i"(off));
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(F.h[1]) : "v"(a1), "i"(off));
  };
  uint32_t sx[FM];
  const uint32_t ea = lb + kE + (uint32_t)r * 4u;

  constexpr int kAhead = 3;            // groups that weight tiles are loaded ahead
  Frag F[4];
  Wt wr[4];
  uint32_t sw = 0;
  // Group c in slab z = c % 4. Its loads are spread one to a fragment, so that no wave stands before a full queue with
  // products to issue: the eight of a weight tile to come over the first fragments, the slab c + 3 over the ones from FB
  // on. There the next slab has landed for this wave once only the loads after its last one are outstanding (a whole group's
  // 8 + P and this group's so far), and the barrier makes every wave's part visible and ends every read of the slab before,
  // which group c + 3 refills.
  auto group = [&](int c, auto jc) {
    constexpr int j = decltype(jc)::value;
    using z_next = std::integral_constant<int, (j + 1) % 4>;
    Wt& w = wr[j];
    Wt& wn = wr[(j + kAhead) % 4];
    auto frag = [&](auto fc) {
      constexpr int f = decltype(fc)::value;
      if constexpr (f == FB) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(vmcnt_wait(8 + P + FB * kWper));
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (f + 3 < FM) rd(F[(f + 3) % 4], std::integral_constant<int, j>{}, std::integral_constant<int, f + 3>{});
      else rd(F[(f + 3) % 4], z_next{}, std::integral_constant<int, f + 3 - FM>{});
      if constexpr (f * kWper < 8)
        each<kWper>([&](auto ic) { load_w(wn, c + kAhead, std::integral_constant<int, f * kWper + decltype(ic)::value>{}); });
      if constexpr (f == FB && j == 1) issue_e(c / 4 + 1);
      if constexpr (f >= FB)
        each<kXper>([&](auto ic) {
          constexpr int p = (f - FB) * kXper + decltype(ic)::value;
          if constexpr (p < P) issue_x(c + 3, std::integral_constant<int, (j + 3) % 4>{}, std::integral_constant<int, p>{});
        });
      Frag& X0 = F[f % 4];
      asm volatile("s_waitcnt lgkmcnt(6)" : "+v"(X0.h[0]), "+v"(X0.h[1]));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 4; ++n)
        mfma8_in_place<j>(acc[f][n], cat8(w.v[n][0], w.v[n][1]), cat8(X0.h[0], X0.h[1]), sw, sx[f]);
      __builtin_amdgcn_sched_barrier(0);
    };
    each<FM>(frag);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  // this part's groups: the same number for each of the slice's `fours` times four; the last ones may be past the last group
  const int per = fours / WK * 4, g0 = (int)blockIdx.y * fours * 4 + part * per;
  issue_e(g0 / 4);
  each<P>([&](auto pc) { issue_x(g0, I0{}, pc); });
  each<kAhead>([&](auto gc) { each<8>([&](auto ic) { load_w(wr[decltype(gc)::value], g0 + decltype(gc)::value, ic); }); });
  each<P>([&](auto pc) { issue_x(g0 + 1, I1{}, pc); });
  each<P>([&](auto pc) { issue_x(g0 + 2, I2{}, pc); });
  __builtin_amdgcn_sched_barrier(0);
  // the first two slabs: the count at the first group's barrier takes loads of a whole group for granted that are not there
  __builtin_amdgcn_s_waitcnt(vmcnt_wait(P));
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  rd(F[0], I0{}, I0{});
  rd(F[1], I0{}, I1{});
  rd(F[2], I0{}, I2{});
  int c = g0;
  do {                  // at least once: no way around the loop, on which the sums would be moved
    // the four groups' exponents: the word of every row that this lane has a fragment of, and the weight block's
    __builtin_amdgcn_sched_barrier(0);
    const uint32_t at = ea + (uint32_t)(c / 4 & 1) * (TM * 4);
    each<FM>([&](auto fc) {
      const uint32_t a = at;
      uint32_t& s = sx[decltype(fc)::value];
      asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(s) : "v"(a), "i"(decltype(fc)::value * 64));
    });
    sw = sew[c < G ? c / 4 : Ge / 4 - 1];
    asm volatile("" : "+v"(sw));
#pragma unroll
    for (int f = 0; f < FM; f += 4)
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(sx[f]), "+v"(sx[f + 1]), "+v"(sx[f + 2]), "+v"(sx[f + 3]));
    __builtin_amdgcn_sched_barrier(0);
    // groups past the last have weights of zero: no branches, across which the compiler would move the products
    group(c, I0{});
    group(c + 1, I1{});
    group(c + 2, I2{});
    group(c + 3, I3{});
    c += 4;
  } while (c < g0 + per);
  // no direct load may still be writing LDS, and no written-out read a register, when the block goes on; the last products
  // are written before their sums are read
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int f = 0; f < FM; ++f) asm volatile("" : "+a"(acc[f][0]), "+a"(acc[f][1]), "+a"(acc[f][2]), "+a"(acc[f][3]));   // not before
  __builtin_amdgcn_sched_barrier(0);
  // Results leave through LDS, in loops: written out element by element they are more instructions than the products, which
  // every launch fetches anew (about 4 us).
  __syncthreads();
  // (the lane's place anew: held over the loop it would cost registers that the loop has not got)
  const int el = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), eq = el >> 4, er = el & 15;
  const auto fin = end();
  using Fin = std::remove_const_t<decltype(fin)>;
  if constexpr (Fin::kRows) {
    // The sums leave through LDS as fp32, fragment by fragment (16 columns of 16 rows; a row's place among its 16 is XORed by
    // the column's, so that reads along a row spread over the banks), 16 FC rows at a time; then 16 lanes take a row of 128 columns,
    // eight each, and end it, four such rows at a time. A lane keeps its columns, so that sums over rows stay in it. What the rows'
    // ends have to read is loaded four rows ahead.
    constexpr int FC = WK == 1 ? FM / 2 : FM, kWaves = 512 / TN, kStep = 4 * kWaves, kTurns = 16 * FC / kStep;
    static_assert(TN % 128 == 0 && kTurns % 4 == 0 && 4 * FC * 4096 <= (int)sizeof(lds));
    f4_t* const all = reinterpret_cast<f4_t*>(lds);
    const int cg = wave / kWaves, at0 = (wave % kWaves) * 4 + eq;
    const int64_t col = n0 + 128 * cg + 8 * er;
    typename Fin::Lane lane8;
    fin.begin(lane8, m0 + at0, kStep, col);
    const int todo = fin.todo();
    // a lane's two fours of a row: wave column and fragment column of its eight columns; rows kStep apart stand in one fragment, or
    // at the same place of the next
    const int pn = (er & 7) >> 1, pq = (er & 1) * 2, pw = 2 * cg + (er >> 3);
    const f4_t* from[16 / kStep][2];
#pragma unroll
    for (int v = 0; v < 16 / kStep; ++v)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        from[v][k] = all + (pw * FC * 4 + pn) * 64 + (pq + k) * 16 + ((at0 + kStep * v) ^ ((pn * 4 + pq + k) ^ (pw & 1)));
    const auto rows_end = [&](auto whole, int left) __attribute__((always_inline)) {      // `left` rows from this lane's next one on
      constexpr bool W = decltype(whole)::value;
      typename Fin::In in[4];
      fin.template load_rows<W>(in, lane8, todo, kStep, left);
#pragma unroll 1
      for (int t = 0; t < kTurns; t += 4, left -= 4 * kStep) {
        float f[4][8];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const f4_t v = from[b % (16 / kStep)][k][(kStep * t / 16 + kStep * b / 16) * 256];
#pragma unroll
            for (int e = 0; e < 4; ++e) f[b][4 * k + e] = v[e];
          }
        typename Fin::In next[4];
        if (t + 4 < kTurns) fin.template load_rows<W>(next, lane8, todo, kStep, left - 4 * kStep);
        __builtin_amdgcn_sched_barrier(0);
        fin.template end_rows<W>(lane8, in, todo, kStep, left, f);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < 4; ++b) in[b] = next[b];
      }
    };
    const bool whole = rows == TM && n0 + TN <= N;
    each<FM / FC>([&](auto hc) {
      constexpr int h = decltype(hc)::value;
      if constexpr (h > 0) __syncthreads();
#pragma unroll
      for (int f = 0; f < FC; ++f) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < 4; ++n)
          all[((wave * FC + f) * 4 + n) * 64 + eq * 16 + (er ^ ((n * 4 + eq) ^ (wi & 1)))] = acc[FC * h + f][n];
      }
      __syncthreads();
      if constexpr (WK > 1) {      // the parts' sums, added in part order into the first's place
#pragma unroll 1
        for (int i = part; i < FM * 4; i += WK) {
          f4_t v = all[(wi * FM * 4 + i) * 64 + el];
#pragma unroll
          for (int k = 1; k < WK; ++k) v += all[((k * WN + wi) * FM * 4 + i) * 64 + el];
          all[(wi * FM * 4 + i) * 64 + el] = v;
        }
        __syncthreads();
      }
      const int left = rows - 16 * FC * h - at0;
      if (whole) rows_end(std::true_type{}, left);
      else rows_end(std::false_type{}, left);
    });
    // sums over the tile's rows: the four row places of a wave, then the waves of a column group in wave order
    if (fin.sums_wanted()) {
      float* const s = reinterpret_cast<float*>(lds);
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = lane8.s[e];
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
        if (eq == 0) s[wave * 128 + 8 * er + e] = v;
      }
      __syncthreads();
      const int t = wave * 64 + el;
      if (t < TN && n0 + t < N) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) v += s[((t >> 7) * kWaves + k) * 128 + (t & 127)];
        fin.put_sum(m0 / TM, n0 + t, N, v);
      }
    }
  } else if constexpr (WK == 1) {
    constexpr int DT = Fin::kType;
    // 16-bit results of the wave's columns, 128 bytes a row, 16-byte slots XOR-swizzled by the row; whole rows leave
    uint8_t* const mine = lds + (uint32_t)wave * (TM * 128);
#pragma unroll
    for (int f = 0; f < FM; ++f) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 4; ++n)
        *reinterpret_cast<u32x2_t*>(mine + (16 * f + er) * 128 + (((2 * n + (eq >> 1)) ^ (er & 7)) * 16) + (eq & 1) * 8) =
            u32x2_t{to_16<DT>(acc[f][n][0]) | to_16<DT>(acc[f][n][1]) << 16, to_16<DT>(acc[f][n][2]) | to_16<DT>(acc[f][n][3]) << 16};
    }
    const int64_t col = n0 + 64 * wi + 8 * (el & 7);
    const int cols = N - col < 8 ? (int)(N - col) : 8;
#pragma unroll 2
    for (int row = el >> 3; row < rows; row += 8) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(mine + row * 128 + (((el & 7) ^ (row & 7)) * 16));
      uint16_t* y = fin.Y + (m0 + row) * fin.ldy + col;
      if (cols == 8) {
        __builtin_memcpy(y, &v, 16);
      } else {
        for (int e = 0; e < cols; ++e) y[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
      }
    }
  } else {
    // the parts' fp32 sums, added in part order; part p finishes fragments p, p + WK, ...
    f4_t* all = reinterpret_cast<f4_t*>(lds);
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int n = 0; n < 4; ++n) all[((wave * FM + f) * 4 + n) * 64 + el] = acc[f][n];
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < FM / WK * 4; ++i) {
      const int f = (i >> 2) * WK + part, n = i & 3;
      f4_t v = all[((wi * FM + f) * 4 + n) * 64 + el];
#pragma unroll
      for (int k = 1; k < WK; ++k) v += all[(((k * WN + wi) * FM + f) * 4 + n) * 64 + el];
      const int row = 16 * f + er;
      const int64_t col = n0 + 64 * wi + 16 * n + 4 * eq;
      if (row < rows && col < N) {
        if (sums) *reinterpret_cast<f4_t*>(sums + ((int64_t)blockIdx.y * M + m0 + row) * ((N + 3) & ~3) + col) = v;
        else fin.four(m0 + row, col, N - col, v);
      }
    }
  }
#endif
}

// ------------------------------------------------------------------------------------- host
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The kernels for a product and what each is thought to take, in microseconds. A tile kernel: a fixed part (launch, first
// loads, last stores), then per group of its part of the reduction `alone` where its blocks are few and `full` where they
// fill the chip (by power and caches), for as many rounds of blocks as there are; not less than the weight's bytes take. The
// constants are fitted to each kernel's times over 126 sizes (M 33 to 4096, N 512 to 28672, K 1024 to 28672; within 5 to 14 %
// of them); picking by them is 0.7 % above the best of the six on average there, 31 % at worst (64 x 28672 x 8192: 52 us
// against 40).
struct TileKind {
  int fm, wn, blocks;      // 16 fm rows, 64 wn columns, 4 / wn parts; blocks that run at once
  double fixed, alone, full;
};
constexpr TileKind kTiles[] = {{16, 4, 256, 10.7, 0.93, 1.48}, {12, 4, 256, 10.8, 0.70, 1.15}, {8, 4, 256, 10.1, 0.54, 0.90},
                               {8, 2, 256, 9.3, 0.57, 1.10},   {4, 2, 512, 8.2, 0.35, 1.33},   {4, 1, 256, 7.2, 0.57, 1.02}};
double tile_time(const TileKind& k, int64_t M, int64_t N, int64_t G, int slices) {
  const int wk = 4 / k.wn;
  const int64_t T = cdiv(M, 16 * k.fm) * cdiv(N, 64 * k.wn) * slices, steps = cdiv(cdiv(G, 4), wk * slices) * 4;
  const int64_t rounds = T / k.blocks, rest = T % k.blocks;
  const double t = rounds * k.full + (rest ? k.alone + (k.full - k.alone) * rest / k.blocks : 0);
  const double sum = slices > 1 ? 3.5 + 2.0 * slices * M * N * 4 / 4e6 : 0;
  return k.fixed + std::max(steps * t, (double)N * G * 128 / 6.0e6) + sum;
}

// The kernel for a product: k_linear8_few with `few` fragments of rows, or tile kernel `kind` over slices of the reduction of
// `fours` times four groups.
struct Plan {
  int few, kind, slices, fours;
  size_t bytes;       // the slices' sums
};
// `narrow`: what tiles of 64 columns cost besides, in microseconds.
Plan plan(int64_t M, int64_t N, int64_t K, double narrow = 0) {
  const int64_t G = q8_row(K) / 128, F = cdiv(G, 4);
  Plan p{0, 0, 1, 0, 0};
  double best = 1e30;
  for (int i = 0; i < 6; ++i) {
    const TileKind& k = kTiles[i];
    const int64_t T = cdiv(M, 16 * k.fm) * cdiv(N, 64 * k.wn);
    // slices where the reduction is in parts already, as long as their blocks run at once
    for (int s = 1; s == 1 || (k.wn < 4 && s * T <= k.blocks && s * (4 / k.wn) <= F && s <= 32); s += s < 4 ? 1 : s / 2) {
      const double t = tile_time(k, M, N, G, s) + (k.wn == 1 && s == 1 ? narrow : 0);
      if (t < best) {
        best = t;
        p.kind = i;
        p.slices = s;
      }
    }
  }
  // (64 x 1024 x 28672 in 16 slices 12 us and 3 for their sum, unsliced 73; 512 x 512 x 28672 27 against 40, 1024 x 1024 x 28672
  // 43 against 60)
  // The few kernel: the weight's bytes, for more rows X's too (two tiles and 32 rows read as many of X as of the weight, one
  // and 64 four times as many), and not less than its 16 groups at a time take where few blocks share a long reduction.
  const double w = (double)N * G * 128, turns = (double)cdiv(G, 16);
  if (M <= 16 && std::max(4 + w * (1 + 0.013 * M) / 6.5e6, 4.5 + (0.75 + 0.035 * M) * turns) < best) p.few = 1;
  else if (M > 16 && M <= 32 && std::max(7 + 2 * w / 8.6e6, 5 + 2.5 * turns) < best) p.few = 2;
  else if (M > 32 && M <= 64 && std::max(6 + 5 * w / 6e6, 5 + 4.2 * turns) < best) p.few = 4;
  const int wk = 4 / kTiles[p.kind].wn;
  p.fours = (int)(cdiv(F, p.slices * wk) * wk);
  p.slices = p.few ? 1 : (int)cdiv(F, p.fours);
  if (p.slices > 1) p.bytes = (size_t)p.slices * (size_t)M * (size_t)((N + 3) & ~int64_t(3)) * 4;
  return p;
}

size_t round256(size_t x) { return (x + 255) & ~size_t(255); }
size_t code_bytes(int64_t M, int64_t K) { return round256((size_t)M * (size_t)q8_row(K)); }

int check_sizes(int xdtype, int64_t M, int64_t N, int64_t K) {
  if (xdtype != SLIM_F16 && xdtype != SLIM_BF16 && xdtype != SLIM_F32 && xdtype != SLIM_Q8_E4M3) return SLIM_EDTYPE;
  if (M < 0 || N < 1 || K < 1 || N > kMaxRow8 || K > kMaxRow8) return SLIM_ESHAPE;
  if (M > (xdtype == SLIM_Q8_E4M3 ? kMaxGroups8 : kMaxQuant8) / (q8_row(K) / 128) || M > kMaxGroups8 / 128) return SLIM_EUNSUPPORTED;
  if (cdiv(M, 64) * cdiv(N, 64) >= (int64_t(1) << 31)) return SLIM_EUNSUPPORTED;      // tiles are counted in 32 bits
  return SLIM_OK;
}

}  // namespace
