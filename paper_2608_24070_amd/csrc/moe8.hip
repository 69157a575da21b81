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
// Logits of RT rows and ET experts a block: a lane takes eight consecutive columns of each 512, its four waves the 512s in turn; sums
// over lanes, then over waves in order. fp32 throughout: products of two 16-bit values are exact. X: 3 for 8-bit rows.
template <int XT, int WT, int RT, int ET>
__global__ void __launch_bounds__(256)
k_route_logits(const void* __restrict__ X, const uint8_t* __restrict__ xe, int64_t ldx, const void* __restrict__ Wr, int64_t ldw, int64_t M,
               int K, int E, float* __restrict__ logits) {
  __shared__ float part[4][RT * ET];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int eb = (E + ET - 1) / ET;
  const int64_t rb = blockIdx.x / eb, m0 = rb * RT;
  const int e0 = (int)(blockIdx.x - rb * eb) * ET;
  float acc[RT][ET] = {};
  for (int c = 8 * (wave * 64 + lane); c < K; c += 8 * 256) {
    float w[ET][8], x[RT][8];
#pragma unroll
    for (int e = 0; e < ET; ++e) load8<WT>(Wr, (int64_t)(e0 + e < E ? e0 + e : E - 1) * ldw + c, K - c, w[e]);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int64_t m = m0 + r < M ? m0 + r : M - 1;
      if constexpr (XT == SLIM_Q8_E4M3) {
        const u32x2_t v = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint8_t*>(X) + m * q8_row(K) + c);
        const float s = q8_pow2(xe[m * q8_exp_row(K) + (c >> 7)]);
        q8_values4(v[0], s, x[r]);
        q8_values4(v[1], s, x[r] + 4);
      } else {
        load8<XT>(X, m * ldx + c, K - c, x[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[r][e] = __builtin_fmaf(x[r][i], w[e][i], acc[r][e]);
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int e = 0; e < ET; ++e) {
      float v = acc[r][e];
#pragma unroll
      for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
      if (lane == 0) part[wave][r * ET + e] = v;
    }
  __syncthreads();
  const int t = threadIdx.x;
  if (t < RT * ET && m0 + t / ET < M && e0 + t % ET < E)
    logits[(m0 + t / ET) * E + e0 + t % ET] = part[0][t] + part[1][t] + part[2][t] + part[3][t];
}

// fp32 as integers in the same order (-0 below +0: made one before).
SLIM_DEV uint32_t ordered(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A wave per row, experts lane + 64 i: the largest logit that is left, the lowest expert that has it, `top` times. A NaN counts as the
// least there and leaves all the row's weights NaN.
__global__ void __launch_bounds__(256)
k_route_top(const float* __restrict__ logits, int64_t M, int E, int top, int renorm, int32_t* __restrict__ ids, float* __restrict__ weights) {
  constexpr int N = kExperts / 64;
  const int lane = threadIdx.x & 63;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= M) return;                                           // whole waves
  float v[N];
  uint32_t key[N];                                              // 0: taken, or no expert
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = lane + 64 * i;
    v[i] = e < E ? logits[m * E + e] : 0.f;
    key[i] = e < E ? (v[i] == v[i] ? ordered(v[i]) : 1u) : 0u;
    big = max(big, key[i]);
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
// The picked experts in order of number, and the rows that picked each with their weights, in order of row. A row that names an expert
// twice is there once, with both weights; a number outside 0 .. E - 1 is nowhere.
struct Table {
  int experts;                       // that were picked
  int expert[kExperts], start[kExperts + 1];
  int row[kTokens * kTop];
  float weight[kTokens * kTop];
};

__global__ void __launch_bounds__(512)
k_moe_table(const int32_t* __restrict__ ids, const float* __restrict__ weights, int M, int top, int E, Table* __restrict__ t) {
  constexpr int P = kTokens * kTop;
  typedef int i32x4_t __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(16))) int id[P];
  __shared__ float weight[P];
  __shared__ int sums[2][8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pairs = M * top;
  for (int i = tid; i < P; i += 512) {
    const int e = i < pairs ? ids[i] : -1;
    id[i] = e >= 0 && e < E ? e : -1;
    weight[i] = i < pairs ? weights[i] : 0.f;
  }
  __syncthreads();
  // a pair whose expert is in its row once more before it goes; the first one takes the weights
  int keep[P / 512];
  float total[P / 512];
#pragma unroll
  for (int k = 0; k < P / 512; ++k) {
    const int i = tid + 512 * k;
    keep[k] = id[i];
    total[k] = weight[i];
    if (i < pairs) {
      const int j = i % top, end = i - j + top;
      for (int o = i - j; o < i; ++o)
        if (id[o] == keep[k]) keep[k] = -1;
      for (int o = i + 1; o < end; ++o)
        if (id[o] == keep[k]) total[k] += weight[o];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < P / 512; ++k) {
    id[tid + 512 * k] = keep[k];
    weight[tid + 512 * k] = total[k];
  }
  __syncthreads();
  // a thread an expert: how many pairs name it
  const int fours = (pairs + 3) / 4, me = tid < E ? tid : -2;
  const i32x4_t* const id4 = reinterpret_cast<const i32x4_t*>(id);
  int n = 0;
#pragma unroll 8
  for (int i = 0; i < fours; ++i) {
    const i32x4_t v = id4[i];
    n += (v[0] == me) + (v[1] == me) + (v[2] == me) + (v[3] == me);
  }
  // places of experts and of their rows: sums over the threads up to this one
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
  for (int w = 0; w < wave; ++w) {
    a += sums[0][w];
    b += sums[1][w];
  }
  if (n > 0) {
    t->expert[a - 1] = tid;
    t->start[a] = b;
    int p = b - n;
#pragma unroll 4
    for (int i = 0; i < fours; ++i) {
      const i32x4_t v = id4[i];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (v[k] == me) {
          t->row[p] = (4 * i + k) / top;
          t->weight[p++] = weight[4 * i + k];
        }
    }
  }
  if (tid == 511) t->experts = a;
  if (tid == 0) t->start[0] = 0;
}

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
template <int XT>
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

// h = act(gate x) * (up x) of the rows that picked expert `slot`: a block takes 16 columns of h, its eight waves the reduction's groups of
// 128 in turn. Weight tiles go straight from memory to registers, two groups of a wave in flight; the rows' values come from L2.
// h leaves as the sum of two bf16 values, 16 significant bits in fp32's range: hi [pairs][F up to 128], then lo.
// GATED: whether there is an up. (A template's parameter: with a branch on w.up between the gate's products and the reads of their
// results the compiler leaves out the wait states that the way past the up's products needs.)
template <int XT, bool GATED>
__global__ void __launch_bounds__(512)
k_moe_up(const uint8_t* __restrict__ X, const uint8_t* __restrict__ xe, int64_t ldx, Experts w, const Table* __restrict__ t,
         uint16_t* __restrict__ hi, uint16_t* __restrict__ lo, int tiles) {
  constexpr int AT = XT == SLIM_Q8_E4M3 ? 1 : XT, FM = kTokens / 16, U = 2, T = GATED ? 2 : 1;
  __shared__ f4_t part[8][T * FM][64];
  const int slot = blockIdx.x / tiles;
  if (slot >= t->experts) return;
  const int e = t->expert[slot], p0 = t->start[slot], n = t->start[slot + 1] - p0;
  const int64_t tile = blockIdx.x - (int64_t)slot * tiles, Ft = (w.F + 15) / 16, Fp = q8_row(w.F);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
  const int K = (int)w.D, G = (int)(q8_row(K) / 128), Ge = (G + 3) & ~3, fm = (n + 15) / 16;
  f4_t acc[T][FM];
#pragma unroll
  for (int k = 0; k < T; ++k)
#pragma unroll
    for (int f = 0; f < FM; ++f) acc[k][f] = f4_t{0.f, 0.f, 0.f, 0.f};
  if (tile < Ft) {
    const int64_t at = ((int64_t)e * Ft + tile) * G * 2048 + lane * 16, ea = ((int64_t)e * ((w.F + 127) / 128) + tile / 8) * Ge;
    const uint8_t* const wp[2] = {w.gate + at, GATED ? w.up + at : nullptr};
    const uint8_t* const we[2] = {w.gate_e + ea, GATED ? w.up_e + ea : nullptr};
    const uint8_t* xp[FM];
    const uint8_t* xs[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
      const bool in = 16 * f + r < n;
      const int64_t m = in ? t->row[p0 + 16 * f + r] : 0;
      xp[f] = !in ? nullptr : XT == SLIM_Q8_E4M3 ? X + m * G * 128 + 32 * q : X + 2 * m * ldx;
      xs[f] = XT == SLIM_Q8_E4M3 ? xe + m * Ge : nullptr;
    }
    for (int g = wave; g < G; g += 8 * U) {
      u32x4_t c[U][T][2];
      float s[U][T];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + 8 * u < G)
#pragma unroll
          for (int k = 0; k < T; ++k) {
#pragma unroll
            for (int h = 0; h < 2; ++h) c[u][k][h] = *reinterpret_cast<const u32x4_t*>(wp[k] + (int64_t)(g + 8 * u) * 2048 + 1024 * h);
            s[u][k] = q8_pow2(we[k][g + 8 * u]);
          }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + 8 * u < G) {
          b8_t wv[T][4];
#pragma unroll
          for (int k = 0; k < T; ++k) widen<AT>(c[u][k], 1.f, wv[k]);
#pragma unroll
          for (int f = 0; f < FM; ++f)
            if (f < fm) {
              b8_t x[4];
              if constexpr (XT == SLIM_Q8_E4M3) {
                u32x4_t xc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                float xsc = 1.f;
                if (xp[f]) {
                  xc[0] = *reinterpret_cast<const u32x4_t*>(xp[f] + (g + 8 * u) * 128);
                  xc[1] = *reinterpret_cast<const u32x4_t*>(xp[f] + (g + 8 * u) * 128 + 16);
                  xsc = q8_pow2(xs[f][g + 8 * u]);
                }
                widen<1>(xc, xsc, x);
              } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = x_eight<XT>(xp[f], (g + 8 * u) * 128 + 32 * q + 8 * i, K);
              }
#pragma unroll
              for (int k = 0; k < T; ++k) {
                f4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i) d = mfma_of<AT>(wv[k][i], x[i], d);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[k][f][i] = __builtin_fmaf(d[i], s[u][k], acc[k][f][i]);
              }
            }
        }
    }
  }
#pragma unroll
  for (int f = 0; f < FM; ++f)
    if (f < fm)
#pragma unroll
      for (int k = 0; k < T; ++k) part[wave][T * f + k][lane] = acc[k][f];
  __syncthreads();
  if (wave < fm) {
    f4_t a = part[0][T * wave][lane], b = part[0][T * wave + T - 1][lane];
#pragma unroll
    for (int k = 1; k < 8; ++k) {
      a += part[k][T * wave][lane];
      if constexpr (GATED) b += part[k][T * wave + 1][lane];
    }
    if (16 * wave + r < n) {
      float h[4];
      with_act(w.act, [&](auto A) {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = act_value<decltype(A)::value>(a[i]);
      });
      u32x2_t vh, vl;
      uint32_t bh[4], bl[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = 16 * tile + 4 * q + i < w.F ? (GATED ? h[i] * b[i] : h[i]) : 0.f;
        bh[i] = to_bf16(v);
        const float left = v - __builtin_bit_cast(float, bh[i] << 16);
        bl[i] = __builtin_fabsf(left) < __builtin_inff() ? to_bf16(left) : 0u;      // of an infinite or NaN value nothing is left
      }
      vh = u32x2_t{bh[0] | bh[1] << 16, bh[2] | bh[3] << 16};
      vl = u32x2_t{bl[0] | bl[1] << 16, bl[2] | bl[3] << 16};
      const int64_t to = (int64_t)(p0 + 16 * wave + r) * Fp + 16 * tile + 4 * q;
      *reinterpret_cast<u32x2_t*>(hi + to) = vh;
      *reinterpret_cast<u32x2_t*>(lo + to) = vl;
    }
  }
}

// y = sum over the picked experts of weight * (down h): a block takes 16 columns of y and one of `parts` parts of all experts'
// groups of 128; its waves take consecutive ones, and add each expert's results to sums of their own in LDS, which are added in wave
// order. With one part y leaves (with the residual), else its fp32 sums.
template <int DT>
__global__ void __launch_bounds__(512)
k_moe_down(const uint16_t* __restrict__ hi, const uint16_t* __restrict__ lo, Experts w, const Table* __restrict__ t, int M, int parts,
           float* __restrict__ sums, const uint16_t* __restrict__ res, int64_t ldres, uint16_t* __restrict__ Y, int64_t ldy) {
  constexpr int FM = kTokens / 16, U = 4;
  __shared__ __attribute__((aligned(16))) float all[8 * kTokens * 16];          // [8 waves][M][16]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
  const int tile = blockIdx.x / parts, part = blockIdx.x - tile * parts;
  const int G = (int)(q8_row(w.F) / 128), Ge = (G + 3) & ~3;
  const int64_t Dt = (w.D + 15) / 16, Db = (w.D + 127) / 128, Fp = (int64_t)G * 128;
  float* const mine = all + wave * M * 16;
  for (int i = lane; i < M * 4; i += 64) *reinterpret_cast<f4_t*>(mine + 4 * i) = f4_t{0.f, 0.f, 0.f, 0.f};
  const int units = t->experts * G, w8 = part * 8 + wave;              // fewer than 2^25
  const int from = (int)((int64_t)units * w8 / (8 * parts)), to = (int)((int64_t)units * (w8 + 1) / (8 * parts));
  for (int u0 = __builtin_amdgcn_readfirstlane(from), end = __builtin_amdgcn_readfirstlane(to); u0 < end;) {
    const int slot = __builtin_amdgcn_readfirstlane(u0 / G);
    const int g0 = u0 - slot * G, g1 = end - slot * G < G ? end - slot * G : G;
    u0 = slot * G + g1;
    const int e = t->expert[slot], p0 = t->start[slot], n = t->start[slot + 1] - p0, fm = (n + 15) / 16;
    const uint8_t* const wp = w.down + ((int64_t)e * Dt + tile) * G * 2048 + lane * 16;
    const uint8_t* const we = w.down_e + ((int64_t)e * Db + tile / 8) * Ge;
    int ha[FM];                                    // at most 64 top rows of F up to 2^22, in eights: below 2^30
#pragma unroll
    for (int f = 0; f < FM; ++f) ha[f] = 16 * f + r < n ? (int)((int64_t)(p0 + 16 * f + r) * Fp / 8) + 4 * q : -1;
    f4_t acc[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) acc[f] = f4_t{0.f, 0.f, 0.f, 0.f};
    for (int g = g0; g < g1; g += U) {
      u32x4_t c[U][2];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u < g1) {
#pragma unroll
          for (int h = 0; h < 2; ++h) c[u][h] = *reinterpret_cast<const u32x4_t*>(wp + (int64_t)(g + u) * 2048 + 1024 * h);
          s[u] = q8_pow2(we[g + u]);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u < g1) {
          b8_t wv[4];
          widen<1>(c[u], 1.f, wv);
#pragma unroll
          for (int f = 0; f < FM; ++f)
            if (f < fm) {
              f4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                u32x4_t a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
                if (ha[f] >= 0) {
                  a = reinterpret_cast<const u32x4_t*>(hi)[(int64_t)(ha[f] + (g + u) * 16 + i)];
                  b = reinterpret_cast<const u32x4_t*>(lo)[(int64_t)(ha[f] + (g + u) * 16 + i)];
                }
                d = mfma_of<1>(wv[i], __builtin_bit_cast(b8_t, a), d);
                d = mfma_of<1>(wv[i], __builtin_bit_cast(b8_t, b), d);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[f][i] = __builtin_fmaf(d[i], s[u], acc[f][i]);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < FM; ++f)
      if (16 * f + r < n) {                        // an expert's rows are distinct
        f4_t* const a = reinterpret_cast<f4_t*>(mine + t->row[p0 + 16 * f + r] * 16 + 4 * q);
        const float k = t->weight[p0 + 16 * f + r];
        *a += acc[f] * k;
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < M * 16; i += 512) {
    float v = all[i];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += all[k * M * 16 + i];
    const int64_t m = i >> 4, col = (int64_t)tile * 16 + (i & 15);
    if (col >= w.D) continue;
    if (parts > 1) {
      sums[((int64_t)part * M + m) * w.D + col] = v;
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

struct MoePlan {
  int parts;
  size_t table, h, sums;
};
MoePlan moe_plan(int64_t M, int64_t D, int64_t F, int64_t top) {
  MoePlan p;
  const int64_t tiles = cdiv(D, 16);
  p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(8, 256 / tiles));
  p.table = round256(sizeof(Table));
  p.h = round256((size_t)(M * top * q8_row(F) * 2));
  p.sums = p.parts > 1 ? round256((size_t)(p.parts * M * D * 4)) : 0;
  return p;
}

template <int XT, int WT>
void launch_logits(const void* X, const uint8_t* xe, int64_t ldx, const void* Wr, int64_t ldw, int64_t M, int64_t K, int E, float* logits,
                   hipStream_t s) {
  SlimKernelTimer timer("route_logits", s);
  if (M >= 8) {
    SLIM_LAUNCH(timer, (k_route_logits<XT, WT, 8, 4>), dim3((unsigned)(cdiv(M, 8) * cdiv(E, 4))), dim3(256), s, X, xe, ldx, Wr, ldw, M, (int)K, E,
                logits);
  } else {
    SLIM_LAUNCH(timer, (k_route_logits<XT, WT, 1, 1>), dim3((unsigned)(M * E)), dim3(256), s, X, xe, ldx, Wr, ldw, M, (int)K, E, logits);
  }
}
template <int XT>
void launch_logits(int wdtype, const void* X, const uint8_t* xe, int64_t ldx, const void* Wr, int64_t ldw, int64_t M, int64_t K, int E,
                   float* logits, hipStream_t s) {
  if (wdtype == SLIM_F16) launch_logits<XT, 0>(X, xe, ldx, Wr, ldw, M, K, E, logits, s);
  else if (wdtype == SLIM_BF16) launch_logits<XT, 1>(X, xe, ldx, Wr, ldw, M, K, E, logits, s);
  else launch_logits<XT, 2>(X, xe, ldx, Wr, ldw, M, K, E, logits, s);
}

}  // namespace

extern "C" int slim_route_workspace(int64_t M, int64_t E, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  if (M < 0 || E < 1) return SLIM_ESHAPE;
  if (E > kExperts || M > (int64_t(1) << 23) / E) return SLIM_EUNSUPPORTED;      // blocks of 256 threads in one launch
  *bytes = (size_t)M * (size_t)E * 4;
  return SLIM_OK;
}

extern "C" int slim_route(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t K, int64_t ldx, const void* Wr, int wdtype,
                          int64_t E, int64_t ldw, int top, int renorm, int32_t* ids, float* weights, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = slim_route_workspace(M, E, &need);
  if (rc != SLIM_OK) return rc;
  const bool packed = xdtype == SLIM_Q8_E4M3;
  if ((!packed && !is_float(xdtype)) || !is_float(wdtype)) return SLIM_EDTYPE;
  if (K < 1 || K > kMaxRow8 || ldw < K || (!packed && ldx < K) || top < 1 || top > E) return SLIM_ESHAPE;
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
  SLIM_LAUNCH(timer, k_route_top, dim3((unsigned)cdiv(M, 4)), dim3(256), s, (const float*)logits, M, (int)E, top, renorm, ids, weights);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

extern "C" int slim_moe8_workspace(int64_t M, int64_t D, int64_t F, int64_t E, int top, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  if (M < 0 || D < 1 || F < 1 || E < 1 || top < 1 || D > kMaxRow8 || F > kMaxRow8) return SLIM_ESHAPE;
  if (M > kTokens || E > kExperts || top > kTop) return SLIM_EUNSUPPORTED;
  if (!one_launch(std::min<int64_t>(E, M * top) * (q8_row(F) / 16), 512)) return SLIM_EUNSUPPORTED;
  *bytes = 0;
  if (M == 0) return SLIM_OK;
  const MoePlan p = moe_plan(M, D, F, top);
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
  hipStream_t s = (hipStream_t)stream;
  const MoePlan p = moe_plan(M, D, F, top);
  char* at = reinterpret_cast<char*>(ws);
  Table* t = reinterpret_cast<Table*>(at);
  uint16_t* hi = reinterpret_cast<uint16_t*>(at + p.table);
  uint16_t* lo = reinterpret_cast<uint16_t*>(at + p.table + p.h);
  float* sums = reinterpret_cast<float*>(at + p.table + 2 * p.h);
  const Experts w{gate, gate_exps, up, up_exps, down, down_exps, D, F, (int)E, act};
  {
    SlimKernelTimer timer("moe_table", s);
    SLIM_LAUNCH(timer, k_moe_table, dim3(1), dim3(512), s, ids, weights, (int)M, top, (int)E, t);
  }
  {
    const int tiles = (int)(q8_row(F) / 16);
    const dim3 grid((unsigned)(std::min<int64_t>(E, M * top) * tiles));
    const uint8_t* x = reinterpret_cast<const uint8_t*>(X);
    SlimKernelTimer timer("moe_up", s);
    const auto call = [&](auto xt) {
      constexpr int XT = decltype(xt)::value;
      SLIM_LAUNCH(timer, (up ? k_moe_up<XT, true> : k_moe_up<XT, false>), grid, dim3(512), s, x, xexps, ldx, w, (const Table*)t, hi, lo, tiles);
    };
    if (packed) call(std::integral_constant<int, SLIM_Q8_E4M3>{});
    else if (xdtype == SLIM_F16) call(std::integral_constant<int, SLIM_F16>{});
    else call(std::integral_constant<int, SLIM_BF16>{});
  }
  const uint16_t* res = reinterpret_cast<const uint16_t*>(residual);
  uint16_t* y = reinterpret_cast<uint16_t*>(Y);
  {
    const dim3 grid((unsigned)(cdiv(D, 16) * p.parts));
    SlimKernelTimer timer("moe_down", s);
    SLIM_LAUNCH(timer, (dtype == SLIM_F16 ? k_moe_down<0> : k_moe_down<1>), grid, dim3(512), s, hi, lo, w, (const Table*)t, (int)M, p.parts, sums,
                res, ldres, y, ldy);
  }
  if (p.parts > 1) {
    const dim3 grid((unsigned)cdiv(M * D, 256));
    SlimKernelTimer timer("moe_sum", s);
    SLIM_LAUNCH(timer, (dtype == SLIM_F16 ? k_moe_sum<0> : k_moe_sum<1>), grid, dim3(256), s, (const float*)sums, p.parts, (int)M, D, res, ldres, y,
                ldy);
  }
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
