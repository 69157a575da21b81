// moe8.hip - a router and a layer of experts for a few tokens: slim_route, slim_moe8.
//
// Router: p = softmax(x Wr^T), the `top` largest of each row. Experts: y_i = sum_j w_ij down_e(act(gate_e x_i) * (up_e x_i)), e =
// ids_ij. With a few tokens the picked experts' weights are all that counts: 3 F D bytes of each, read once, against 2 D bytes of
// a token. They are kept as slim_pack8's tiles; activations stay in 16 bits, since the matrix unit has far more room than memory
// gives weights: codes are widened to the activations' type (exact in both) and each group of 128 is scaled in fp32. So neither x
// nor the experts' inner values are rounded to 8 bits.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <type_traits>

#include "slim_act.h"
#include "slim_launch.h"
#include "slim_q8.h"
#include "slim_timing.h"

namespace {

typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));

constexpr int kTokens = 64;          // rows of one call of slim_moe8
constexpr int kExperts = 512, kTop = 16;

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t x) { return (x + 255) & ~size_t(255); }

// ------------------------------------------------------------------------------------- router
// Sums over the lanes of N values each (N a power of two up to 64): lane l ends with value l / (64 / N) of the sum over all lanes. Each step
// gives half of the values to the other half of the lanes, so that N - 1 exchanges do for all, and the last ones for sums.
template <int N, int D = 32>
SLIM_DEV float lanes_sum(float* v, int lane) {
  if constexpr (D == 0) {
    return v[0];
  } else if constexpr (N == 1) {
    v[0] += __shfl_xor(v[0], D, 64);
    return lanes_sum<1, D / 2>(v, lane);
  } else {
    const bool high = lane & D;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float other = __shfl_xor(high ? v[i] : v[N / 2 + i], D, 64);
      v[i] = (high ? v[N / 2 + i] : v[i]) + other;
    }
    return lanes_sum<N / 2, D / 2>(v, lane);
  }
}

// Parts of the logits: ET experts, up to 2 RT rows and 2048 columns a block. A wave takes 512 columns, a lane eight of them, whose router
// values stay in registers while RT rows at a time go by; sums over lanes, then over the block's four waves in order, and
// k_route_top adds the parts. So the router is read once and x comes from L2. fp32 throughout: products of two 16-bit values are exact.
// X: 3 for 8-bit rows.
constexpr int kRouteCols = 2048;
constexpr int route_rows(int rt) { return 2 * rt; }
template <int XT, int WT, int RT, int ET>
__global__ void __launch_bounds__(256)
k_route_logits(const void* __restrict__ X, const uint8_t* __restrict__ xe, int64_t ldx, const void* __restrict__ Wr, int64_t ldw, int64_t M,
               int K, int E, int parts, float* __restrict__ logits) {
  constexpr int N = RT * ET, kRows = route_rows(RT);
  __shared__ float sums[4][kRows * ET];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, eb = (E + ET - 1) / ET;
  const int64_t rb = blockIdx.x / (eb * parts), m0 = rb * kRows;
  const int left = (int)(blockIdx.x - rb * eb * parts), part = left / eb, e0 = (left - part * eb) * ET;
  const int rows = (int)(M - m0 < kRows ? M - m0 : kRows), c = part * kRouteCols + 512 * wave + 8 * lane;
  float w[ET][8];
#pragma unroll
  for (int e = 0; e < ET; ++e) load8<WT>(Wr, (int64_t)(e0 + e < E ? e0 + e : E - 1) * ldw + c, K - c, w[e]);      // zeros past K
  for (int r0 = 0; r0 < rows; r0 += RT) {
    float x[RT][8], acc[N];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int64_t m = m0 + (r0 + r < rows ? r0 + r : rows - 1);
      if constexpr (XT == SLIM_Q8_E4M3) {
        if (c < K) {
          const u32x2_t v = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint8_t*>(X) + m * q8_row(K) + c);
          const float s = q8_pow2(xe[m * q8_exp_row(K) + (c >> 7)]);
          q8_values4(v[0], s, x[r]);
          q8_values4(v[1], s, x[r] + 4);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[r][i] = 0.f;
        }
      } else {
        load8<XT>(X, m * ldx + c, K - c, x[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < ET; ++e) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = __builtin_fmaf(x[r][i], w[e][i], a);
        acc[r * ET + e] = a;
      }
    const float v = lanes_sum<N>(acc, lane);
    const int i = r0 * ET + lane / (64 / N);
    if (lane % (64 / N) == 0 && i < rows * ET) sums[wave][i] = v;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * ET; i += 256) {
    const int e = e0 + i % ET;
    if (e < E) logits[((int64_t)part * M + m0 + i / ET) * E + e] = sums[0][i] + sums[1][i] + sums[2][i] + sums[3][i];
  }
}

// fp32 as integers in the same order (-0 below +0: made one before).
SLIM_DEV uint32_t ordered(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A wave per row, experts lane + 64 i: the largest logit that is left, the lowest expert that has it, `top` times. A NaN counts as the
// least there and leaves all the row's weights NaN.
template <int N>      // 64 N experts at most
__global__ void __launch_bounds__(256)
k_route_top(const float* __restrict__ logits, int parts, int64_t M, int E, int top, int renorm, int32_t* __restrict__ ids,
            float* __restrict__ weights) {
  const int lane = threadIdx.x & 63;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= M) return;                                           // whole waves
  float v[N];
  uint32_t key[N];                                              // 0: taken, or no expert
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = lane + 64 * i;
    v[i] = 0.f;
    if (e < E)
      for (int p = 0; p < parts; ++p) v[i] += logits[((int64_t)p * M + m) * E + e];
    key[i] = e < E ? (v[i] == v[i] ? ordered(v[i]) : 1u) : 0u;
  }
  float most = 0.f, sum = 0.f, mine = 0.f;
  int at = 0;
  for (int j = 0; j < top; ++j) {
    uint32_t k = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) k = max(k, key[i]);
    k = wave_max_u32(k);
    int e = -1;
    float x = 0.f;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
      const uint64_t has = __ballot(key[i] == k);
      if (has) {
        const int l = __builtin_ctzll(has);
        e = l + 64 * i;
        x = __shfl(v[i], l, 64);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane + 64 * i == e) key[i] = 0;
    if (j == 0) most = x;
    if (lane == j) {
      mine = x;
      at = e;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane + 64 * i < E) sum += expf(v[i] - most);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  float p = lane < top ? expf(mine - most) / sum : 0.f;
  if (renorm) {
    float all = p;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d, 64);
    p /= all;
  }
  if (lane < top) {
    ids[m * top + lane] = at;
    weights[m * top + lane] = p;
  }
}

// ------------------------------------------------------------------------------------- who goes where
// The picked experts in order of number, each with a run of places: the rows that picked it with their weights, in order of row. A
// row that names an expert twice is there once, with both weights; a number outside 0 .. E - 1 is nowhere. Slots behind the last
// expert have n = 0.
struct Slot {
  int expert, start, n, pad;
};
struct Table {
  int experts, pad[3];
  Slot slot[kExperts];
  int row[kTokens * kTop];
  float weight[kTokens * kTop];
};

// One block: a thread a pair of row and expert (two at most), then a thread an expert, which has its rows as 64 bits: how many they are
// and how many lie before one of them is a count of bits.
static_assert(kTokens <= 64 && kExperts <= 512 && kTokens * kTop == 2 * 512);
__global__ void __launch_bounds__(512)
k_moe_table(const int32_t* __restrict__ ids, const float* __restrict__ weights, int M, int top, int E, Table* __restrict__ t) {
  constexpr int P = kTokens * kTop;
  __shared__ int id[P];
  __shared__ float weight[P];
  __shared__ uint32_t rows[2][kExperts];
  __shared__ int first[kExperts];
  __shared__ int sums[2][8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pairs = M * top;
  rows[0][tid] = rows[1][tid] = 0;
#pragma unroll
  for (int k = 0; k < P / 512; ++k) {
    const int i = tid + 512 * k, e = i < pairs ? ids[i] : -1;
    id[i] = e >= 0 && e < E ? e : -1;
    weight[i] = i < pairs ? weights[i] : 0.f;
  }
  __syncthreads();
  // of an expert's pairs in one row the first takes all weights
  int mine[P / 512];
  float total[P / 512];
#pragma unroll
  for (int k = 0; k < P / 512; ++k) {
    const int i = tid + 512 * k;
    mine[k] = id[i];
    total[k] = weight[i];
    if (i < pairs && mine[k] >= 0) {
      const int row = i / top, j = i - row * top, end = i - j + top, e = mine[k];
      for (int o = i - j; o < i; ++o)
        if (id[o] == e) mine[k] = -1;
      for (int o = i + 1; o < end; ++o)
        if (id[o] == e) total[k] += weight[o];
      atomicOr(&rows[row >> 5][e], 1u << (row & 31));
    }
  }
  __syncthreads();
  // places of experts and of their runs: sums over the experts up to this one
  const int n = __builtin_popcount(rows[0][tid]) + __builtin_popcount(rows[1][tid]);
  int a = n > 0, b = n;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int pa = __shfl_up(a, d, 64), pb = __shfl_up(b, d, 64);
    if (lane >= d) {
      a += pa;
      b += pb;
    }
  }
  if (lane == 63) {
    sums[0][wave] = a;
    sums[1][wave] = b;
  }
  __syncthreads();
  int experts = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    if (w < wave) {
      a += sums[0][w];
      b += sums[1][w];
    }
    experts += sums[0][w];
  }
  first[tid] = b - n;
  if (n > 0) t->slot[a - 1] = Slot{tid, b - n, n, 0};
  if (tid >= experts) t->slot[tid] = Slot{0, 0, 0, 0};
  if (tid == 0) t->experts = experts;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < P / 512; ++k) {
    const int i = tid + 512 * k;
    if (i < pairs && mine[k] >= 0) {
      const int row = i / top, e = mine[k];
      const uint32_t low = row < 32 ? (1u << row) - 1 : ~0u, high = row < 32 ? 0u : (1u << (row - 32)) - 1;
      const int place = first[e] + __builtin_popcount(rows[0][e] & low) + __builtin_popcount(rows[1][e] & high);
      t->row[place] = row;
      t->weight[place] = total[k];
    }
  }
}

// What a kernel knows of it: the table, or for one row the numbers themselves (a slot for each, its place the slot's own).
struct Picks {
  const Table* t;          // null: one row
  const int32_t* ids;
  const float* weights;
  int top, E;

  SLIM_DEV Slot slot(int s) const {
    if (t) return t->slot[s];
    const int e = ids[s];
    bool good = e >= 0 && e < E;
    for (int o = 0; o < s; ++o) good &= ids[o] != e;
    return Slot{good ? e : 0, s, good ? 1 : 0, 0};
  }
  SLIM_DEV int row(int place) const { return t ? t->row[place] : 0; }
  SLIM_DEV float weight(int place) const {
    if (t) return t->weight[place];
    float w = weights[place];
    for (int o = place + 1; o < top; ++o)
      if (ids[o] == ids[place]) w += weights[o];
    return w;
  }
};

// ------------------------------------------------------------------------------------- experts
// 32 codes of a lane as four operands of eight 16-bit values, times 2^(b - 127) (weights: b = 127, exact).
template <int AT>
SLIM_DEV void widen(const u32x4_t* c, float s, b8_t* o) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t v = c[i >> 2][i & 3];
    if constexpr (AT == 1) {
      const b2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, s, true);
      o[i >> 1][4 * (i & 1)] = lo[0];
      o[i >> 1][4 * (i & 1) + 1] = lo[1];
      o[i >> 1][4 * (i & 1) + 2] = hi[0];
      o[i >> 1][4 * (i & 1) + 3] = hi[1];
    } else {
      const h2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, s, true);
      const u32x2_t w = {bits_of(lo), bits_of(hi)};
      u32x4_t t = __builtin_bit_cast(u32x4_t, o[i >> 1]);
      t[2 * (i & 1)] = w[0];
      t[2 * (i & 1) + 1] = w[1];
      o[i >> 1] = __builtin_bit_cast(b8_t, t);
    }
  }
}
template <int AT>
SLIM_DEV f4_t mfma_of(b8_t a, b8_t b, f4_t c) {
  if constexpr (AT == 1) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  else return mfma16(__builtin_bit_cast(h8_t, a), __builtin_bit_cast(h8_t, b), c);
}

struct Experts {
  const uint8_t *gate, *gate_e, *up, *up_e, *down, *down_e;    // one expert after the other
  int64_t D, F;
  int E, act;
};

// 8 values of a row from column c on, zeros past K; p is null for a row that is not there.
SLIM_DEV b8_t x_eight(const uint8_t* p, int c, int K) {
  u32x4_t v = {0, 0, 0, 0};
  if (p && c < K) {
    if (K - c >= 8) {
      __builtin_memcpy(&v, p + 2 * (int64_t)c, 16);
    } else {
      const uint16_t* t = reinterpret_cast<const uint16_t*>(p) + c;
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < K - c) v[e >> 1] |= (uint32_t)t[e] << (16 * (e & 1));
    }
  }
  return __builtin_bit_cast(b8_t, v);
}

// act(gate x) and up x of one tile of 16 columns for the FM sixteens of a slot's rows, summed over this wave's groups of 128: its weight
// tiles go straight from memory to registers, U groups of a wave in flight with the rows' values for them (from L2).
template <int XT, int T, int FM, int U, int W>
SLIM_DEV void up_groups(const uint8_t* X, const uint8_t* xe, int64_t ldx, const Picks& picks, const Slot& slot, int K,
                        const uint8_t* const* wp, const uint8_t* const* we, int wave, int lane, f4_t (*acc)[T]) {
  constexpr int AT = XT == SLIM_Q8_E4M3 ? 1 : XT;
  const int r = lane & 15, q = lane >> 4, G = (int)(q8_row(K) / 128), Ge = (G + 3) & ~3;
  const uint8_t* xp[FM];
  const uint8_t* xs[FM];
#pragma unroll
  for (int f = 0; f < FM; ++f) {
    const bool in = 16 * f + r < slot.n;
    const int64_t m = in ? picks.row(slot.start + 16 * f + r) : 0;
    xp[f] = !in ? nullptr : XT == SLIM_Q8_E4M3 ? X + m * G * 128 + 32 * q : X + 2 * m * ldx;
    xs[f] = XT == SLIM_Q8_E4M3 ? xe + m * Ge : nullptr;
#pragma unroll
    for (int k = 0; k < T; ++k) acc[f][k] = f4_t{0.f, 0.f, 0.f, 0.f};
  }
  for (int g0 = wave; g0 < G; g0 += W * U) {
    u32x4_t c[U][T][2];
    float s[U][T];
    b8_t x[U][FM][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int g = g0 + W * u;
      if (g < G) {
#pragma unroll
        for (int k = 0; k < T; ++k) {
#pragma unroll
          for (int h = 0; h < 2; ++h) c[u][k][h] = *reinterpret_cast<const u32x4_t*>(wp[k] + (int64_t)g * 2048 + 1024 * h);
          s[u][k] = q8_pow2(we[k][g]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int g = g0 + W * u;
      if (g < G)
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          if constexpr (XT == SLIM_Q8_E4M3) {
            // codes and exponent for now, widened where they are used
            u32x4_t v[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
            u32x4_t e = {127, 0, 0, 0};
            if (xp[f]) {
              v[0] = *reinterpret_cast<const u32x4_t*>(xp[f] + g * 128);
              v[1] = *reinterpret_cast<const u32x4_t*>(xp[f] + g * 128 + 16);
              e[0] = xs[f][g];
            }
            x[u][f][0] = __builtin_bit_cast(b8_t, v[0]);
            x[u][f][1] = __builtin_bit_cast(b8_t, v[1]);
            x[u][f][2] = __builtin_bit_cast(b8_t, e);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[u][f][i] = x_eight(xp[f], g * 128 + 32 * q + 8 * i, K);
          }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g0 + W * u < G) {
        b8_t wv[T][4];
#pragma unroll
        for (int k = 0; k < T; ++k) widen<AT>(c[u][k], 1.f, wv[k]);
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          b8_t xv[4];
          if constexpr (XT == SLIM_Q8_E4M3) {
            const u32x4_t v[2] = {__builtin_bit_cast(u32x4_t, x[u][f][0]), __builtin_bit_cast(u32x4_t, x[u][f][1])};
            widen<1>(v, q8_pow2(__builtin_bit_cast(u32x4_t, x[u][f][2])[0]), xv);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) xv[i] = x[u][f][i];
          }
#pragma unroll
          for (int k = 0; k < T; ++k) {
            f4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) d = mfma_of<AT>(wv[k][i], xv[i], d);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[f][k][i] = __builtin_fmaf(d[i], s[u][k], acc[f][k][i]);
          }
        }
      }
  }
}

// h = act(gate x) * (up x) of the rows that picked the expert of a slot, 16 columns of h a block, the reduction's groups over its four
// waves, whose sums are added through LDS in wave order. h leaves as the sum of two bf16 values, 16 significant bits in fp32's range:
// hi [pairs][F up to 128], then lo. GATED: whether there is an up. (A template's parameter: with a branch on w.up between the gate's
// products and the reads of their results the compiler leaves out the wait states that the way past the up's products needs.)
// Bound by the weights' bytes: 7 rows, 2 of 8 experts, 4096 x 11008 95 to 101 us where 6 of the eight are picked, 123 to 145 where all are (4.9
// to 5.9 TB/s; more where calls on two sets of weights take turns); 8 of 64 of 4096 x 1024 for one row 17 to 19 us (3.9 to 3.5), as one of
// many calls: a block's first loads wait for its slot.
template <int XT, bool GATED>
__global__ void __launch_bounds__(256, 2)
k_moe_up(const uint8_t* __restrict__ X, const uint8_t* __restrict__ xe, int64_t ldx, Experts w, Picks picks, uint16_t* __restrict__ hi,
         uint16_t* __restrict__ lo, int tiles) {
  constexpr int FM = kTokens / 16, T = GATED ? 2 : 1, W = 4;
  __shared__ f4_t part[W][T * FM][64];
  const int at = blockIdx.x / tiles;
  const Slot slot = picks.slot(at);
  if (slot.n == 0) return;
  const int64_t tile = blockIdx.x - (int64_t)at * tiles, Ft = (w.F + 15) / 16, Fp = q8_row(w.F);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
  const int K = (int)w.D, G = (int)(q8_row(K) / 128), Ge = (G + 3) & ~3, fm = (slot.n + 15) / 16;
  if (tile < Ft) {
    const int64_t to = ((int64_t)slot.expert * Ft + tile) * G * 2048 + lane * 16, te = ((int64_t)slot.expert * ((w.F + 127) / 128) + tile / 8) * Ge;
    const uint8_t* const wp[2] = {w.gate + to, GATED ? w.up + to : nullptr};
    const uint8_t* const we[2] = {w.gate_e + te, GATED ? w.up_e + te : nullptr};
    const auto run = [&](auto fc, auto uc) SLIM_INLINE {
      constexpr int F = decltype(fc)::value;
      f4_t acc[F][T];
      up_groups<XT, T, F, decltype(uc)::value, W>(X, xe, ldx, picks, slot, K, wp, we, wave, lane, acc);
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int k = 0; k < T; ++k) part[wave][T * f + k][lane] = acc[f][k];
    };
    using std::integral_constant;
    if (fm == 1) run(integral_constant<int, 1>{}, integral_constant<int, 4>{});
    else if (fm == 2) run(integral_constant<int, 2>{}, integral_constant<int, 2>{});
    else run(integral_constant<int, 4>{}, integral_constant<int, 1>{});
  }
  __syncthreads();
  if (wave < fm && 16 * wave + r < slot.n) {
    float h[4] = {0.f, 0.f, 0.f, 0.f};
    if (tile < Ft) {
      f4_t a = part[0][T * wave][lane], b = part[0][T * wave + T - 1][lane];
#pragma unroll
      for (int k = 1; k < W; ++k) {
        a += part[k][T * wave][lane];
        if constexpr (GATED) b += part[k][T * wave + 1][lane];
      }
      with_act(w.act, [&](auto A) SLIM_INLINE {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = act_value<decltype(A)::value>(a[i]);
      });
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = 16 * tile + 4 * q + i < w.F ? (GATED ? h[i] * b[i] : h[i]) : 0.f;      // zeros up to the group's end
    }
    uint32_t bh[4], bl[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bh[i] = to_bf16(h[i]);
      const float left = h[i] - __builtin_bit_cast(float, bh[i] << 16);
      bl[i] = __builtin_fabsf(left) < __builtin_inff() ? to_bf16(left) : 0u;      // of an infinite or NaN value nothing is left
    }
    const int64_t to = (int64_t)(slot.start + 16 * wave + r) * Fp + 16 * tile + 4 * q;
    *reinterpret_cast<u32x2_t*>(hi + to) = u32x2_t{bh[0] | bh[1] << 16, bh[2] | bh[3] << 16};
    *reinterpret_cast<u32x2_t*>(lo + to) = u32x2_t{bl[0] | bl[1] << 16, bl[2] | bl[3] << 16};
  }
}

// Groups g0 .. g1 of a slot's h times NT tiles of 16 of its expert's down, added with the rows' weights to this wave's sums
// mine [M][16 NT] in LDS. U groups in flight.
template <int NT, int FM, int U>
SLIM_DEV void down_groups(const u32x4_t* hi, const u32x4_t* lo, const Picks& picks, const Slot& slot, int G, int g0, int g1,
                          const uint8_t* wp, const int* next, const uint8_t* we, int lane, float* mine) {
  const int r = lane & 15, q = lane >> 4;
  int ha[FM];                                      // in eights: at most 64 top rows of F up to 2^22, below 2^30
#pragma unroll
  for (int f = 0; f < FM; ++f) ha[f] = 16 * f + r < slot.n ? (slot.start + 16 * f + r) * G * 16 + 4 * q : -1;
  f4_t acc[FM][NT];
#pragma unroll
  for (int f = 0; f < FM; ++f)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[f][n] = f4_t{0.f, 0.f, 0.f, 0.f};
  for (int g = g0; g < g1; g += U) {
    u32x4_t c[U][NT][2], a[U][FM][4], b[U][FM][4];
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u < g1) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) c[u][n][h] = *reinterpret_cast<const u32x4_t*>(wp + (int64_t)(g + u) * 2048 + next[n] + 1024 * h);
        s[u] = q8_pow2(we[g + u]);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u < g1)
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a[u][f][i] = b[u][f][i] = u32x4_t{0, 0, 0, 0};
            if (ha[f] >= 0) {
              a[u][f][i] = hi[(int64_t)(ha[f] + (g + u) * 16 + i)];
              b[u][f][i] = lo[(int64_t)(ha[f] + (g + u) * 16 + i)];
            }
          }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u < g1)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          b8_t wv[4];
          widen<1>(c[u][n], 1.f, wv);
#pragma unroll
          for (int f = 0; f < FM; ++f) {
            f4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              d = mfma_of<1>(wv[i], __builtin_bit_cast(b8_t, a[u][f][i]), d);
              d = mfma_of<1>(wv[i], __builtin_bit_cast(b8_t, b[u][f][i]), d);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[f][n][i] = __builtin_fmaf(d[i], s[u], acc[f][n][i]);
          }
        }
  }
#pragma unroll
  for (int f = 0; f < FM; ++f)
    if (16 * f + r < slot.n) {                     // an expert's rows are distinct
      const int place = slot.start + 16 * f + r;
      float* const row = mine + picks.row(place) * 16 * NT + 4 * q;
      const float k = picks.weight(place);
#pragma unroll
      for (int n = 0; n < NT; ++n) *reinterpret_cast<f4_t*>(row + 16 * n) += acc[f][n] * k;
    }
}

// y = sum over the slots of weight * (down h): a block takes 16 NT columns of y and one of `parts` parts of all slots' groups of 128; its
// W waves take consecutive ones, and add each expert's results to sums of their own in LDS, which are added in wave order. With one
// part y leaves (with the residual), else its fp32 sums. (Eight tiles of a weight share one row of exponents, and NT divides eight.)
// 7 rows, 2 of 8, 4096 x 11008 54 us where 6 of the eight are picked, 69 to 82 where all are (4.4 to 5.2 TB/s), and 4 for the parts' sum; 61 rows,
// 4 of 40, 5120 x 1700, 39 picked, 80 to 90 (3.8 to 4.1); one row, 8 of 64, 4096 x 1024 12.6 (2.7): eight groups a wave, one round of loads.
template <int DT, int NT, int W>
__global__ void __launch_bounds__(64 * W, W == 4 ? 2 : 1)
k_moe_down(const u32x4_t* __restrict__ hi, const u32x4_t* __restrict__ lo, Experts w, Picks picks, int slots, int M, int parts,
           float* __restrict__ sums, const uint16_t* __restrict__ res, int64_t ldres, uint16_t* __restrict__ Y, int64_t ldy) {
  __shared__ __attribute__((aligned(16))) float all[W * kTokens * 16 * NT];          // [W][M][16 NT]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int strip = blockIdx.x / parts, part = blockIdx.x - strip * parts;
  const int G = (int)(q8_row(w.F) / 128), Ge = (G + 3) & ~3;
  const int D = (int)w.D, Dt = (D + 15) / 16, Db = (D + 127) / 128, tile = strip * NT;
  float* const mine = all + wave * M * 16 * NT;
  for (int i = lane; i < M * 4 * NT; i += 64) *reinterpret_cast<f4_t*>(mine + 4 * i) = f4_t{0.f, 0.f, 0.f, 0.f};
  const int used = picks.t ? picks.t->experts : slots;
  int next[NT];                                               // the strip's tiles from its first on; past the last: not stored
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    next[n] = (tile + n < Dt ? n : Dt - 1 - tile) * G * 2048;
    asm volatile("" : "+v"(next[n]));                         // scalar registers are short here
  }
  const int units = used * G, w8 = part * W + wave;           // fewer than 2^25
  const int from = __builtin_amdgcn_readfirstlane((int)((int64_t)units * w8 / (W * parts)));
  const int end = __builtin_amdgcn_readfirstlane((int)((int64_t)units * (w8 + 1) / (W * parts)));
  for (int u0 = from; u0 < end;) {
    const int s = __builtin_amdgcn_readfirstlane(u0 / G);
    const int g0 = u0 - s * G, g1 = end - s * G < G ? end - s * G : G;
    u0 = s * G + g1;
    const Slot slot = picks.slot(s);
    if (slot.n == 0) continue;
    const uint8_t* const wp = w.down + ((int64_t)slot.expert * Dt + tile) * G * 2048 + lane * 16;
    const uint8_t* const we = w.down_e + ((int64_t)slot.expert * Db + tile / 8) * Ge;
    if (slot.n <= 16) down_groups<NT, 1, NT == 1 ? 4 : 2>(hi, lo, picks, slot, G, g0, g1, wp, next, we, lane, mine);
    else      // 32 rows at a time: what an expert has past them reads its weights again, from L2
      for (int done = 0; done < slot.n; done += 32)
        down_groups<NT, 2, NT == 1 ? 2 : 1>(hi, lo, picks, Slot{slot.expert, slot.start + done, slot.n - done, 0}, G, g0, g1, wp, next, we, lane, mine);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < M * 16 * NT; i += 64 * W) {
    float v = all[i];
#pragma unroll
    for (int k = 1; k < W; ++k) v += all[k * M * 16 * NT + i];
    const int64_t m = i / (16 * NT), col = tile * 16 + i % (16 * NT);
    if (col >= D) continue;
    if (parts > 1) {
      sums[((int64_t)part * M + m) * D + col] = v;
    } else {
      if (res) v += load_elem<DT>(res, m * ldres + col);
      store_elem<DT>(Y, m * ldy + col, v);
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(256)
k_moe_sum(const float* __restrict__ sums, int parts, int M, int64_t D, const uint16_t* __restrict__ res, int64_t ldres, uint16_t* __restrict__ Y,
          int64_t ldy) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = M * D;
  if (i >= all) return;
  float v = sums[i];
  for (int k = 1; k < parts; ++k) v += sums[k * all + i];
  const int64_t m = i / D, col = i - m * D;
  if (res) v += load_elem<DT>(res, m * ldres + col);
  store_elem<DT>(Y, m * ldy + col, v);
}

// ------------------------------------------------------------------------------------- host
bool is_16(int t) { return t == SLIM_F16 || t == SLIM_BF16; }
bool is_float(int t) { return is_16(t) || t == SLIM_F32; }
size_t elem(int t) { return t == SLIM_F32 ? 4 : 2; }

// Four tiles of y a block from three rows on, where h, which every strip reads, would cost as much as the weights do (down and its sum: 4
// rows, 2 of 8 experts, 4096 x 11008: 47 us against 61; 16 rows, 4 of 32, 4096 x 2048: 44 against 65; one row, 8 of 64, 4096 x 1024: 14
// against 12.6). Parts of the reduction until 256 blocks of eight waves or 512 of four are there, each wave with eight groups at
// least; for many rows, whose parts' sums count, 256 (64 rows, 4 of 32, 2048 x 2048: 42 us, 53 with 512; 2 of 8, 8192 x 2048: 46, 55).
struct MoePlan {
  int tiles, waves, slots, parts;
  int64_t strips;
  size_t table, h, sums;
};
MoePlan moe_plan(int64_t M, int64_t D, int64_t F, int64_t E, int64_t top) {
  MoePlan p;
  p.slots = (int)(M == 1 ? top : std::min<int64_t>(E, M * top));
  p.tiles = M <= 2 ? 1 : 4;
  p.waves = p.tiles == 1 ? 8 : 4;
  p.strips = cdiv(cdiv(D, 16), p.tiles);
  const int64_t units = p.slots * (q8_row(F) / 128), fill = p.tiles == 4 && M <= 32 ? 512 : 256;
  p.parts = (int)std::max<int64_t>(1, std::min({fill / p.strips, units / (8 * p.waves), int64_t(16)}));
  p.table = M == 1 ? 0 : round256(sizeof(Table));
  p.h = round256((size_t)(M * top * q8_row(F) * 2));
  p.sums = p.parts > 1 ? round256((size_t)(p.parts * M * D * 4)) : 0;
  return p;
}

template <int XT, int WT>
void launch_logits(const void* X, const uint8_t* xe, int64_t ldx, const void* Wr, int64_t ldw, int64_t M, int64_t K, int E, float* logits,
                   hipStream_t s) {
  SlimKernelTimer timer("route_logits", s);
  const int parts = (int)cdiv(K, kRouteCols);
  // few rows: a block for every expert and two of them, which is all latency (7 x 8 x 4096 3.9 us against 7.7); more: the router's values
  // are kept over 16 rows (61 x 250 x 8192, fp32 router: 15 us; over all 61 rows, in a quarter of the blocks, 37; 8192 x 64 x 4096, 156)
  if (M >= 8)
    SLIM_LAUNCH(timer, (k_route_logits<XT, WT, 8, 4>), dim3((unsigned)(cdiv(M, route_rows(8)) * parts * cdiv(E, 4))), dim3(256), s, X, xe, ldx, Wr,
                ldw, M, (int)K, E, parts, logits);
  else
    SLIM_LAUNCH(timer, (k_route_logits<XT, WT, 1, 1>), dim3((unsigned)(cdiv(M, route_rows(1)) * parts * E)), dim3(256), s, X, xe, ldx, Wr, ldw, M,
                (int)K, E, parts, logits);
}
template <int XT>
void launch_logits(int wdtype, const void* X, const uint8_t* xe, int64_t ldx, const void* Wr, int64_t ldw, int64_t M, int64_t K, int E,
                   float* logits, hipStream_t s) {
  if (wdtype == SLIM_F16) launch_logits<XT, 0>(X, xe, ldx, Wr, ldw, M, K, E, logits, s);
  else if (wdtype == SLIM_BF16) launch_logits<XT, 1>(X, xe, ldx, Wr, ldw, M, K, E, logits, s);
  else launch_logits<XT, 2>(X, xe, ldx, Wr, ldw, M, K, E, logits, s);
}

}  // namespace

extern "C" int slim_route_workspace(int64_t M, int64_t E, int64_t K, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  if (M < 0 || E < 1 || K < 1 || K > kMaxRow8) return SLIM_ESHAPE;
  if (E > kExperts || M > int64_t(1) << 32 || !one_launch(cdiv(M, route_rows(8)) * cdiv(K, kRouteCols) * E, 256)) return SLIM_EUNSUPPORTED;
  if (!one_launch(cdiv(M, 4), 256)) return SLIM_EUNSUPPORTED;
  *bytes = (size_t)cdiv(K, kRouteCols) * (size_t)M * (size_t)E * 4;
  return SLIM_OK;
}

extern "C" int slim_route(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t K, int64_t ldx, const void* Wr, int wdtype,
                          int64_t E, int64_t ldw, int top, int renorm, int32_t* ids, float* weights, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = slim_route_workspace(M, E, K, &need);
  if (rc != SLIM_OK) return rc;
  const bool packed = xdtype == SLIM_Q8_E4M3;
  if ((!packed && !is_float(xdtype)) || !is_float(wdtype)) return SLIM_EDTYPE;
  if (ldw < K || (!packed && ldx < K) || top < 1 || top > E) return SLIM_ESHAPE;
  if (top > kTop) return SLIM_EUNSUPPORTED;
  if (M == 0) return SLIM_OK;
  if (!X || (packed && !xexps) || !Wr || !ids || !weights) return SLIM_EINVAL;
  if (!slim_aligned_to(X, packed ? 16 : elem(xdtype)) || !slim_aligned16(xexps) || !slim_aligned_to(Wr, elem(wdtype)) ||
      !slim_aligned_to(ids, 4) || !slim_aligned_to(weights, 4))
    return SLIM_EALIGN;
  if (!ws || ws_bytes < need) return SLIM_EWORKSPACE;
  if (!slim_aligned16(ws)) return SLIM_EALIGN;
  hipStream_t s = (hipStream_t)stream;
  float* logits = reinterpret_cast<float*>(ws);
  if (packed) launch_logits<SLIM_Q8_E4M3>(wdtype, X, xexps, ldx, Wr, ldw, M, K, (int)E, logits, s);
  else if (xdtype == SLIM_F16) launch_logits<SLIM_F16>(wdtype, X, xexps, ldx, Wr, ldw, M, K, (int)E, logits, s);
  else if (xdtype == SLIM_BF16) launch_logits<SLIM_BF16>(wdtype, X, xexps, ldx, Wr, ldw, M, K, (int)E, logits, s);
  else launch_logits<SLIM_F32>(wdtype, X, xexps, ldx, Wr, ldw, M, K, (int)E, logits, s);
  SlimKernelTimer timer("route_top", s);
  SLIM_LAUNCH(timer, (E <= 64 ? k_route_top<1> : E <= 128 ? k_route_top<2> : E <= 256 ? k_route_top<4> : k_route_top<8>),
              dim3((unsigned)cdiv(M, 4)), dim3(256), s, (const float*)logits, (int)cdiv(K, kRouteCols), M, (int)E, top, renorm, ids, weights);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

extern "C" int slim_moe8_workspace(int64_t M, int64_t D, int64_t F, int64_t E, int top, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  if (M < 0 || D < 1 || F < 1 || E < 1 || top < 1 || D > kMaxRow8 || F > kMaxRow8) return SLIM_ESHAPE;
  if (M > kTokens || E > kExperts || top > kTop) return SLIM_EUNSUPPORTED;
  if (!one_launch(std::max<int64_t>(top, std::min<int64_t>(E, M * top)) * (q8_row(F) / 16), 256)) return SLIM_EUNSUPPORTED;
  *bytes = 0;
  if (M == 0) return SLIM_OK;
  const MoePlan p = moe_plan(M, D, F, E, top);
  *bytes = p.table + 2 * p.h + p.sums;
  return SLIM_OK;
}

extern "C" int slim_moe8(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t D, int64_t ldx, int64_t F, int64_t E,
                         const uint8_t* gate, const uint8_t* gate_exps, const uint8_t* up, const uint8_t* up_exps, const uint8_t* down,
                         const uint8_t* down_exps, int act, const int32_t* ids, const float* weights, int top, const void* residual,
                         int64_t ldres, void* Y, int dtype, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = slim_moe8_workspace(M, D, F, E, top, &need);
  if (rc != SLIM_OK) return rc;
  const bool packed = xdtype == SLIM_Q8_E4M3;
  if ((!packed && !is_16(xdtype)) || !is_16(dtype)) return SLIM_EDTYPE;
  if (act < SLIM_ACT_NONE || act > SLIM_ACT_SILU) return SLIM_EINVAL;
  if ((!packed && ldx < D) || ldy < D || (residual && ldres < D)) return SLIM_ESHAPE;
  if (M == 0) return SLIM_OK;
  if (!X || (packed && !xexps) || !gate || !gate_exps || !up != !up_exps || !down || !down_exps || !ids || !weights || !Y) return SLIM_EINVAL;
  if (!slim_aligned_to(X, packed ? 16 : 2) || !slim_aligned16(xexps) || !slim_aligned16(gate) || !slim_aligned16(gate_exps) ||
      !slim_aligned16(up) || !slim_aligned16(up_exps) || !slim_aligned16(down) || !slim_aligned16(down_exps) || !slim_aligned_to(ids, 4) ||
      !slim_aligned_to(weights, 4) || !slim_aligned_to(residual, 2) || !slim_aligned_to(Y, 2))
    return SLIM_EALIGN;
  if (!ws || ws_bytes < need) return SLIM_EWORKSPACE;
  if (!slim_aligned16(ws)) return SLIM_EALIGN;
  // X is read before the launch that writes Y; the residual in that launch, element for element by the lane that writes there, and with
  // one row ids and weights, by every block
  const SlimRows picked{ids, 1, M * top * 4, 0}, weighed{weights, 1, M * top * 4, 0};
  if (!slim_may_write({{Y, M, 2 * D, 2 * ldy}}, {{residual, M, 2 * D, 2 * ldres}}, {picked, weighed})) return SLIM_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  const MoePlan p = moe_plan(M, D, F, E, top);
  char* at = reinterpret_cast<char*>(ws);
  Table* t = reinterpret_cast<Table*>(at);
  uint16_t* hi = reinterpret_cast<uint16_t*>(at + p.table);
  uint16_t* lo = reinterpret_cast<uint16_t*>(at + p.table + p.h);
  float* sums = reinterpret_cast<float*>(at + p.table + 2 * p.h);
  const Experts w{gate, gate_exps, up, up_exps, down, down_exps, D, F, (int)E, act};
  const Picks picks{M == 1 ? nullptr : t, ids, weights, top, (int)E};
  if (M > 1) {
    SlimKernelTimer timer("moe_table", s);
    SLIM_LAUNCH(timer, k_moe_table, dim3(1), dim3(512), s, ids, weights, (int)M, top, (int)E, t);
  }
  {
    const int tiles = (int)(q8_row(F) / 16);
    const dim3 grid((unsigned)((int64_t)p.slots * tiles));
    const uint8_t* x = reinterpret_cast<const uint8_t*>(X);
    SlimKernelTimer timer("moe_up", s);
    const auto call = [&](auto xt) {
      constexpr int XT = decltype(xt)::value;
      SLIM_LAUNCH(timer, (up ? k_moe_up<XT, true> : k_moe_up<XT, false>), grid, dim3(256), s, x, xexps, ldx, w, picks, hi, lo, tiles);
    };
    if (packed) call(std::integral_constant<int, SLIM_Q8_E4M3>{});
    else if (xdtype == SLIM_F16) call(std::integral_constant<int, SLIM_F16>{});
    else call(std::integral_constant<int, SLIM_BF16>{});
  }
  const uint16_t* res = reinterpret_cast<const uint16_t*>(residual);
  uint16_t* y = reinterpret_cast<uint16_t*>(Y);
  {
    const dim3 grid((unsigned)(p.strips * p.parts));
    SlimKernelTimer timer("moe_down", s);
    const auto call = [&](auto kernel, int waves) {
      SLIM_LAUNCH(timer, kernel, grid, dim3(64 * waves), s, reinterpret_cast<const u32x4_t*>(hi), reinterpret_cast<const u32x4_t*>(lo), w, picks,
                  p.slots, (int)M, p.parts, sums, res, ldres, y, ldy);
    };
    if (p.tiles == 1) call(dtype == SLIM_F16 ? k_moe_down<0, 1, 8> : k_moe_down<1, 1, 8>, 8);
    else call(dtype == SLIM_F16 ? k_moe_down<0, 4, 4> : k_moe_down<1, 4, 4>, 4);
  }
  if (p.parts > 1) {
    const dim3 grid((unsigned)cdiv(M * D, 256));
    SlimKernelTimer timer("moe_sum", s);
    SLIM_LAUNCH(timer, (dtype == SLIM_F16 ? k_moe_sum<0> : k_moe_sum<1>), grid, dim3(256), s, (const float*)sums, p.parts, (int)M, D, res, ldres, y,
                ldy);
  }
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
