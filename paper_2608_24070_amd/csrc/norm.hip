// norm.hip - layer norm and RMS norm over rows, forward (slim_norm) and backward (slim_norm_bwd).
//
//   forward   mu = mean_k x, v = mean_k (x - mu)^2, rstd = (v + eps)^(-1/2), y = (x - mu) rstd gamma + beta
//             (RMS norm: mu = 0)
//   backward  xh = (x - mu) rstd, t = dy gamma, dx = rstd (t - mean_k t - xh mean_k (t xh)) (RMS norm: without
//             mean_k t), dgamma = sum_m dy xh, dbeta = sum_m dy
//
// Every row is read once and stays in registers between its sums and its result; a block takes rows block by block, so
// that gamma, beta and the column sums of the backward stay in registers too, and loads the next row before it works on
// the present one. All arithmetic is fp32; y and dx are rounded once. Sums have a fixed order, so results repeat bit for
// bit. Bound by HBM. Figures are of a launch by itself with its operands from memory, unless they say otherwise.
#include <hip/hip_runtime.h>
#include <algorithm>

#include "slim_launch.h"
#include "slim_q8.h"
#include "slim_timing.h"

namespace {

constexpr int kQ8 = SLIM_Q8_E4M3;   // the element type of rows in 8 bits

// Eight consecutive elements of a row as they are stored.
template <int DT> struct Raw8 { u32x4_t v; };
template <> struct Raw8<2> { f4_t a, b; };
template <> struct Raw8<kQ8> { u32x2_t c; float s; };

// Rows of one operand: element type, row stride in elements, exponents (8-bit rows, whose stride is whole groups).
struct RowsOf {
  const void* p;
  const uint8_t* exps;
  int64_t ld;
};

// Vector `col` .. `col` + 7 of a row, zeros past its end. RAG: rows may end inside a vector (K % 8 != 0); the kernels are
// built apart for it, since the tests of single elements cost the others their scalar registers. FILL: values of the row past its
// end (a vector's first, or the row's; rows in 8 bits that end inside a vector have zeros there); whole vectors and 8-bit rows
// are then loaded without a test (8-bit rows, 8192 x 8192: both launches 73 us, with it 93).
template <int DT, bool RAG, bool FILL = false>
SLIM_DEV Raw8<DT> load_raw8(const RowsOf& r, int64_t row, int64_t col, int64_t K) {
  Raw8<DT> o;
  if constexpr (FILL) col = col < K ? col : 0;
  int n = RAG ? (int)(K - col) : FILL || col < K ? 8 : 0;
  const int64_t i = row * r.ld + col;
  if constexpr (RAG && !(FILL && DT == kQ8)) asm volatile("" : "+v"(n));      // compared here, not held as masks over a caller's loop
  if constexpr (DT == kQ8) {
    // rows are padded to whole groups with zeros
    o.c = u32x2_t{0, 0};
    o.s = 0.f;
    if (FILL || n > 0) {
      o.c = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint8_t*>(r.p) + i);
      o.s = q8_pow2(r.exps[row * ((r.ld + 511) / 512 * 4) + col / 128]);
    }
  } else if constexpr (DT == 2) {
    if (RAG) {
      float f[8];
      if (!FILL || n >= 8) {
        load8<2>(r.p, i, n, f);
      } else {
        const float* p = reinterpret_cast<const float*>(r.p) + i;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = p[e < n ? e : 0];
      }
      o.a = f4_t{f[0], f[1], f[2], f[3]};
      o.b = f4_t{f[4], f[5], f[6], f[7]};
    } else {
      o.a = o.b = f4_t{0.f, 0.f, 0.f, 0.f};
      if (n > 0) {
        const float* p = reinterpret_cast<const float*>(r.p) + i;
        __builtin_memcpy(&o.a, p, 16);
        __builtin_memcpy(&o.b, p + 4, 16);
      }
    }
  } else {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(r.p) + i;
    if (!RAG || n >= 8) {
      o.v = u32x4_t{0, 0, 0, 0};
      if (RAG || n > 0) __builtin_memcpy(&o.v, p, 16);
    } else if (FILL) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o.v[e] = (uint32_t)p[2 * e < n ? 2 * e : 0] | (uint32_t)p[2 * e + 1 < n ? 2 * e + 1 : 0] << 16;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o.v[e] = (2 * e < n ? (uint32_t)p[2 * e] : 0u) | (2 * e + 1 < n ? (uint32_t)p[2 * e + 1] << 16 : 0u);
    }
  }
  return o;
}

template <int DT>
SLIM_DEV void values8(const Raw8<DT>& o, float* f) {
  if constexpr (DT == kQ8) {
    q8_values4(o.c[0], o.s, f);
    q8_values4(o.c[1], o.s, f + 4);
  } else if constexpr (DT == 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[e] = o.a[e];
      f[4 + e] = o.b[e];
    }
  } else {
    act8_to_f(o.v, DT == 1, f);
  }
}

// xh = (x - mu) rstd of eight elements, the difference first: x rstd - mu rstd in one operation would leave a rounding of
// mu rstd, which in rows far from zero with little or no variance passes xh itself. (The second operation for each element
// hides behind memory: 8192 x 8192 in bf16 82.8 us for both launches before, 83.0 with it.)
// Past a row's end dy is zero, but xh has to be finite for a sum over the row to leave it out, and of x = 0 it would be
// -mu rstd: so x is loaded with FILL there.
template <int DT>
SLIM_DEV void xhat8(const Raw8<DT>& o, float mu, float rstd, float* f) {
  if constexpr (DT == kQ8) {
    q8_values4(o.c[0], 1.f, f);
    q8_values4(o.c[1], 1.f, f + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = fmaf(f[e], o.s, -mu) * rstd;
  } else {
    values8<DT>(o, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (f[e] - mu) * rstd;
  }
}

// What FILL leaves of rows in 8 bits that end inside a vector (RAG): the codes from the n-th on are set to the first one's, in
// rows whose mu rstd is infinite (or NaN), few if any.
template <int DT, bool RAG>
SLIM_DEV void fill8(Raw8<DT>& o, int n) {
  if constexpr (DT == kQ8 && RAG) {
    if (n < 8) {
      const uint64_t keep = (uint64_t(1) << (8 * n)) - 1, first = (uint64_t)((o.c[0] & 255u) * 0x01010101u);
      const uint64_t c = (((uint64_t)o.c[1] << 32 | o.c[0]) & keep) | ((first << 32 | first) & ~keep);
      o.c = u32x2_t{(uint32_t)c, (uint32_t)(c >> 32)};
    }
  }
}
template <int DT, bool RAG>
SLIM_DEV bool needs_fill8(float mu, float rstd) { return DT == kQ8 && RAG && !(fabsf(mu * rstd) < __builtin_inff()); }

// Eight parameters (gamma, beta) as fp32; `none` where there are none.
template <bool RAG>
SLIM_DEV void params8(const void* p, int dt, int64_t col, int64_t K, float none, float* f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = none;
  if (!p || col >= K) return;
  const int64_t n = RAG ? K - col : 8;
  if (dt == 2) load8<2>(p, col, n, f);
  else if (dt == 1) load8<1>(p, col, n, f);
  else load8<0>(p, col, n, f);
}

// Sum over the wave's lanes, the same in every lane: rotations within rows of 16 lanes, then the four rows.
SLIM_DEV float wave_sum(float v) {
#define SLIM_ADD_ROR(n) v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + n, 0xF, 0xF, false))
  SLIM_ADD_ROR(1);
  SLIM_ADD_ROR(2);
  SLIM_ADD_ROR(4);
  SLIM_ADD_ROR(8);
#undef SLIM_ADD_ROR
  const int i = __builtin_bit_cast(int, v);
  const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 0)), b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 16));
  const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 32)), d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 48));
  return (a + b) + (c + d);
}

// Two sums over the T threads that share a row; `turn` alternates from row to row, so that one barrier a row is enough:
// a thread that is a row ahead writes the other half of `part`, and none can be two ahead.
template <int T>
SLIM_DEV f2_t row_sums(float a, float b, f2_t (*part)[T / 64], int turn) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (T == 64) {
    return f2_t{a, b};
  } else {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[turn][wave] = f2_t{a, b};
    __syncthreads();
    f2_t s = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < T / 64; ++w) s += part[turn][w];
    return s;
  }
}

// Largest bits over aligned groups of 16 lanes (one group of 128 values at 8 a lane).
SLIM_DEV uint32_t row16_max_u32(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
}

// Eight results of a row to memory; in 8 bits the sixteen lanes of a group agree on its exponent first. `col` counts whole
// lanes, so the groups' lanes past K take part with zeros; the last lanes of a row write the padding.
template <int DT, bool RAG>
SLIM_DEV void store_row8(void* y, uint8_t* exps, int64_t row, int64_t ld, int64_t col, int64_t K, float* f) {
  if constexpr (DT == kQ8) {
    uint32_t m = 0;
    int n = (int)(K - col);
    asm volatile("" : "+v"(n));       // compared here, not held as masks over a caller's loop
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = (RAG ? e : 0) < n ? f[e] : 0.f;
      m = max(m, q8_abs(f[e]));
    }
    const uint32_t b = q8_exponent(row16_max_u32(m));
    const int64_t Kp = q8_row(K), Ge = q8_exp_row(K);
    const int in = n + (int)(Kp - K);                 // columns from here to the end of the last group
    if (in > 0) {
      const float s = q8_inverse(b);
      const u32x2_t c = {q8_codes4(f[0], f[1], f[2], f[3], s), q8_codes4(f[4], f[5], f[6], f[7], s)};
      *reinterpret_cast<u32x2_t*>(reinterpret_cast<uint8_t*>(y) + row * Kp + col) = c;
      const int sub = (int)(col & 127) / 8;
      uint8_t* e = exps + row * Ge + col / 128;
      if (sub == 0) *e = (uint8_t)b;
      else if (in <= 128 && sub <= (int)(Ge - Kp / 128)) e[sub] = 0;      // the row's last word ends in zeros
    }
  } else {
    int n = RAG ? (int)(K - col) : 8;
    if constexpr (RAG) asm volatile("" : "+v"(n));
    if (col < K) store8<DT>(y, row * ld + col, n, f);
  }
}

// ------------------------------------------------------------------------------------- forward
struct NormArgs {
  RowsOf x;
  const void* gamma;
  const void* beta;
  int pdt;              // type of gamma and beta
  bool rms;
  float eps;
  int64_t M, K;
  void* y;
  int64_t ldy;
  uint8_t* yexps;
  float* mean;
  float* rstd;
};

// Rows of up to 8 T V elements, T threads a row, V vectors of 8 a thread. Each wave sums its part of the row about its
// own mean, and the waves' (count, mean, squares) are joined exactly as if about the row's mean: one barrier a row, and no
// cancellation for rows far from zero. Means are quotients, not products with 1 / K, so that a row of one value has that
// value as its mean wherever its sum is exact, and results of beta. HOLD: gamma and beta stay in registers from row to row;
// AHEAD: the next row is loaded before the present one is worked on (both as registers allow).
// Bound by memory: 8192 x 8192 in bf16 49.1 us (5.5 TB/s read and written), to 8 bits 57.2 us (3.5 TB/s); 2047 x 5120 in
// fp16 16.5 us, 11.7 where calls follow each other; one row of 4096 6.4 us, which is a launch and two trips to memory, 3.1 as one
// of many in a graph.
template <int DT, int YT, int T, int V, bool HOLD, bool AHEAD, bool RAG>
__global__ void __launch_bounds__(T == 64 ? 256 : T)
k_norm(NormArgs a) {
  constexpr int kRows = T == 64 ? 4 : 1, kWaves = T / 64, H = HOLD ? V : 1;
  __shared__ f2_t part[2][kWaves];
  __shared__ float count[kWaves];      // elements of the row that a wave holds
  const int t = threadIdx.x % T;
  const int64_t first = (int64_t)blockIdx.x * kRows + threadIdx.x / T, step = (int64_t)gridDim.x * kRows;
  float gm[H][8], bt[H][8];
  Raw8<DT> nx[V];
  int mine = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t col = (int64_t)(v * T + t) * 8;
    if (AHEAD && first < a.M) nx[v] = load_raw8<DT, RAG>(a.x, first, col, a.K);
    if constexpr (HOLD) {
      params8<RAG>(a.gamma, a.pdt, col, a.K, 1.f, gm[v]);
      params8<RAG>(a.beta, a.pdt, col, a.K, 0.f, bt[v]);
    }
    const int64_t n = a.K - (int64_t)(v * T + (t & ~63)) * 8;
    mine += n <= 0 ? 0 : n > 512 ? 512 : (int)n;
  }
  if (T > 64 && (t & 63) == 0) count[t >> 6] = (float)mine;
  const float held = mine ? (float)mine : 1.f, inv_k = 1.f / (float)a.K;
  int turn = 0;
  for (int64_t row = first; row < a.M; row += step, turn ^= 1) {
    float x[V][8];
    if (!AHEAD)
#pragma unroll
      for (int v = 0; v < V; ++v) nx[v] = load_raw8<DT, RAG>(a.x, row, (int64_t)(v * T + t) * 8, a.K);
#pragma unroll
    for (int v = 0; v < V; ++v) values8<DT>(nx[v], x[v]);
    if (AHEAD && row + step < a.M)
#pragma unroll
      for (int v = 0; v < V; ++v) nx[v] = load_raw8<DT, RAG>(a.x, row + step, (int64_t)(v * T + t) * 8, a.K);
    float mu = 0.f, sq = 0.f;
    if (!a.rms) {
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[v][e];
      mu = wave_sum(s) / held;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      int n = (int)(a.K - (v * T + t) * 8);
      asm volatile("" : "+v"(n));        // compared here, not held as masks over the loop
      const float m = n > 0 ? mu : 0.f;
      if (RAG) {
        // the last vector's places past the row take the mean, the ones of lanes past it stay zero: no square either way
#pragma unroll
        for (int e = 1; e < 8; ++e) x[v][e] = e < n ? x[v][e] : m;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = x[v][e] - m;
        sq = fmaf(d, d, sq);
      }
    }
    sq = wave_sum(sq);
    if constexpr (T > 64) {
      if ((t & 63) == 0) part[turn][t >> 6] = f2_t{mu, sq};
      __syncthreads();
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) sum = fmaf(count[i], part[turn][i][0], sum);
      mu = sum / (float)a.K;
      sq = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float d = part[turn][i][0] - mu;
        sq += fmaf(count[i] * d, d, part[turn][i][1]);
      }
    }
    const float rstd = 1.f / sqrtf(fmaf(sq, inv_k, a.eps));
    if (t == 0) {
      if (a.mean) a.mean[row] = mu;
      a.rstd[row] = rstd;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t col = (int64_t)(v * T + t) * 8;
      const int h = HOLD ? v : 0;
      if constexpr (!HOLD) {
        params8<RAG>(a.gamma, a.pdt, col, a.K, 1.f, gm[0]);
        params8<RAG>(a.beta, a.pdt, col, a.K, 0.f, bt[0]);
      }
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fmaf((x[v][e] - mu) * rstd, gm[h][e], bt[h][e]);
      store_row8<YT, RAG>(a.y, a.yexps, row, a.ldy, col, a.K, y);
    }
  }
}

// Longer rows: one block a row reads it three times (mean, squares, result), the later times from the caches. Also ragged
// rows past 16384, where a vector's tests for the row's end cost the kernel above its scalar registers: 2048 x 28671 in
// bf16 100 us (28672 in registers: 65.5 us).
template <int DT, int YT>
__global__ void __launch_bounds__(1024)
k_norm_long(NormArgs a) {
  __shared__ f2_t part[2][16];
  const int64_t row = blockIdx.x;
  const int64_t end = q8_row(a.K);     // whole groups, so that the lanes of one stay together
  float mu = 0.f;
  if (!a.rms) {
    float s = 0.f;
    for (int64_t col = threadIdx.x * 8; col < a.K; col += 8192) {
      float x[8], p = 0.f;
      values8<DT>(load_raw8<DT, true>(a.x, row, col, a.K), x);
#pragma unroll
      for (int e = 0; e < 8; ++e) p += x[e];
      s += p;
    }
    mu = row_sums<1024>(s, 0.f, part, 0)[0] / (float)a.K;
  }
  float s = 0.f;
  for (int64_t col = threadIdx.x * 8; col < a.K; col += 8192) {
    float x[8], p = 0.f;
    values8<DT>(load_raw8<DT, true>(a.x, row, col, a.K), x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = col + e < a.K ? x[e] - mu : 0.f;
      p = fmaf(d, d, p);
    }
    s += p;
  }
  const float rstd = 1.f / sqrtf(row_sums<1024>(s, 0.f, part, 1)[0] / (float)a.K + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mu;
    a.rstd[row] = rstd;
  }
  for (int64_t col = threadIdx.x * 8; col < end; col += 8192) {
    float x[8], g[8], b[8];
    values8<DT>(load_raw8<DT, true>(a.x, row, col, a.K), x);
    params8<true>(a.gamma, a.pdt, col, a.K, 1.f, g);
    params8<true>(a.beta, a.pdt, col, a.K, 0.f, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf((x[e] - mu) * rstd, g[e], b[e]);
    store_row8<YT, true>(a.y, a.yexps, row, a.ldy, col, a.K, x);
  }
}

// ------------------------------------------------------------------------------------- backward
struct NormBwdArgs {
  RowsOf dy, x;
  const void* gamma;
  int pdt;
  const float* mean;    // null: RMS norm
  const float* rstd;
  int64_t M, K;
  void* dx;
  int64_t lddx;
  float* part;          // column sums of each block: [blocks][2][K] (dgamma, dbeta)
  float* dgamma;
  float* dbeta;
};

// As k_norm: T threads a row, V vectors a thread; dgamma's and dbeta's sums over the block's rows stay in registers and
// leave as one row of partial sums a block (k_norm_cols adds those in block order). Rows of up to 8192 take 256 threads of
// four vectors rather than 512 of two: two blocks share a CU and do not wait at one barrier (8192 x 8192 in bf16 79.0 and
// 96.7 us). That is 5.1 TB/s; k_norm_cols takes another 5.8 us. From 8 bits 66.6 us (5.1 TB/s). 8192 x 4096 37.2 + 4.6 (from 8
// bits 35.1), 2047 x 5120 in fp16 24.4 + 4.1, 333 x 1000 from 8 bits 8.2 + 7.0 (both launches in a graph 8.0). RMS norms take
// dbeta's sums along: a row of registers and half of k_norm_cols' reading.
template <int DT, int XT, int T, int V, bool HOLD, bool AHEAD, bool RAG>
__global__ void __launch_bounds__(T == 64 ? 256 : T)
k_norm_bwd(NormBwdArgs a) {
  constexpr int kRows = T == 64 ? 4 : 1;
  __shared__ f2_t part[2][T / 64];
  __shared__ float join[kRows > 1 ? 3 : 1][kRows > 1 ? 2 : 1][kRows > 1 ? V * T * 8 : 1];
  const int t = threadIdx.x % T;
  const int64_t first = (int64_t)blockIdx.x * kRows + threadIdx.x / T, step = (int64_t)gridDim.x * kRows;
  constexpr int H = HOLD ? V : 1;
  float gm[H][8], dg[V][8], db[V][8];
  Raw8<DT> ny[V];
  Raw8<XT> nx[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t col = (int64_t)(v * T + t) * 8;
    if (AHEAD && first < a.M) {
      ny[v] = load_raw8<DT, RAG>(a.dy, first, col, a.K);
      nx[v] = load_raw8<XT, RAG, true>(a.x, first, col, a.K);
    }
    if constexpr (HOLD) params8<RAG>(a.gamma, a.pdt, col, a.K, 1.f, gm[v]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[v][e] = db[v][e] = 0.f;
  }
  const float inv_k = 1.f / (float)a.K;
  int turn = 0;
  for (int64_t row = first; row < a.M; row += step, turn ^= 1) {
    const float mu = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
    Raw8<DT> y[V];
    Raw8<XT> x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (AHEAD) {
        y[v] = ny[v];
        x[v] = nx[v];
      } else {
        y[v] = load_raw8<DT, RAG>(a.dy, row, (int64_t)(v * T + t) * 8, a.K);
        x[v] = load_raw8<XT, RAG, true>(a.x, row, (int64_t)(v * T + t) * 8, a.K);
      }
    }
    if (AHEAD && row + step < a.M)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        ny[v] = load_raw8<DT, RAG>(a.dy, row + step, (int64_t)(v * T + t) * 8, a.K);
        nx[v] = load_raw8<XT, RAG, true>(a.x, row + step, (int64_t)(v * T + t) * 8, a.K);
      }
    if (needs_fill8<XT, RAG>(mu, rstd))
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int n = (int)a.K - (v * T + t) * 8;
        fill8<XT, RAG>(x[v], n > 0 ? n : (int)a.K);          // vectors past the end hold the row's first
      }
    float st = 0.f, sx = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float d[8], h[8];
      values8<DT>(y[v], d);
      xhat8<XT>(x[v], mu, rstd, h);
      const int g = HOLD ? v : 0;
      if constexpr (!HOLD) params8<RAG>(a.gamma, a.pdt, (int64_t)(v * T + t) * 8, a.K, 1.f, gm[0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float tt = d[e] * gm[g][e];     // zero past K
        st += tt;
        sx = fmaf(tt, h[e], sx);
        dg[v][e] = fmaf(d[e], h[e], dg[v][e]);
        db[v][e] += d[e];
      }
    }
    const f2_t sums = row_sums<T>(st, sx, part, turn);
    const float mt = a.mean ? sums[0] * inv_k : 0.f, mx = sums[1] * inv_k;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float d[8], h[8];
      values8<DT>(y[v], d);
      xhat8<XT>(x[v], mu, rstd, h);
      const int g = HOLD ? v : 0;
      if constexpr (!HOLD) params8<RAG>(a.gamma, a.pdt, (int64_t)(v * T + t) * 8, a.K, 1.f, gm[0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = rstd * fmaf(-mx, h[e], fmaf(d[e], gm[g][e], -mt));
      store_row8<DT, RAG>(a.dx, nullptr, row, a.lddx, (int64_t)(v * T + t) * 8, a.K, d);
    }
  }
  if constexpr (kRows > 1) {
    // the block's four rows of sums, in wave order
    const int w = threadIdx.x / T;
    if (w > 0) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          join[w - 1][0][(v * 8 + e) * T + t] = dg[v][e];
          join[w - 1][1][(v * 8 + e) * T + t] = db[v][e];
        }
    }
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        for (int i = 0; i < 3; ++i) {
          dg[v][e] += join[i][0][(v * 8 + e) * T + t];
          db[v][e] += join[i][1][(v * 8 + e) * T + t];
        }
  }
  // one block: its sums are the gradients
  float* const og = gridDim.x == 1 ? a.dgamma : a.part + (int64_t)blockIdx.x * 2 * a.K;
  float* const ob = gridDim.x == 1 ? a.dbeta : a.part + ((int64_t)blockIdx.x * 2 + 1) * a.K;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t col = (int64_t)(v * T + t) * 8;
    if (col < a.K) {
      if (og) store8<2>(og, col, RAG ? a.K - col : 8, dg[v]);
      if (ob) store8<2>(ob, col, RAG ? a.K - col : 8, db[v]);
    }
  }
}

// Longer rows, second kernel: dx, one block a row, which reads it twice (400 x 65536 in bf16: 41.7 us). The column sums of
// such rows have a kernel of their own (24.3 us there).
template <int DT, int XT>
__global__ void __launch_bounds__(1024)
k_norm_bwd_long(NormBwdArgs a) {
  __shared__ f2_t part[2][16];
  const int64_t row = blockIdx.x;
  const float mu = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
  float st = 0.f, sx = 0.f;
  for (int64_t col = threadIdx.x * 8; col < a.K; col += 8192) {
    float d[8], h[8], g[8], p = 0.f, q = 0.f;
    values8<DT>(load_raw8<DT, true>(a.dy, row, col, a.K), d);
    Raw8<XT> x = load_raw8<XT, true, true>(a.x, row, col, a.K);
    if (needs_fill8<XT, true>(mu, rstd)) fill8<XT, true>(x, (int)(a.K - col));
    xhat8<XT>(x, mu, rstd, h);
    params8<true>(a.gamma, a.pdt, col, a.K, 1.f, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float tt = d[e] * g[e];
      p += tt;
      q = fmaf(tt, h[e], q);
    }
    st += p;
    sx += q;
  }
  const f2_t sums = row_sums<1024>(st, sx, part, 0);
  const float mt = a.mean ? sums[0] / (float)a.K : 0.f, mx = sums[1] / (float)a.K;
  for (int64_t col = threadIdx.x * 8; col < a.K; col += 8192) {
    float d[8], h[8], g[8];
    values8<DT>(load_raw8<DT, true>(a.dy, row, col, a.K), d);
    xhat8<XT>(load_raw8<XT, true>(a.x, row, col, a.K), mu, rstd, h);
    params8<true>(a.gamma, a.pdt, col, a.K, 1.f, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = rstd * fmaf(-mx, h[e], fmaf(d[e], g[e], -mt));
    store_row8<DT, true>(a.dx, nullptr, row, a.lddx, col, a.K, d);
  }
}

// The same for whole vectors and rows of up to 32768: the row stays in registers between its sums and its result. 2048 x 28672
// in bf16 76 us, 4.6 TB/s, after 53 for the column sums (where calls follow each other 121 for all three launches); 3221 x 20832 in
// fp32 159 us after 116. Read twice, dx took 80 us for 72, and 196 for 165. (The column sums would fit beside 16-bit and 8-bit rows
// of up to 28672 with seven vectors a thread, and gamma read anew; that has not been built.)
template <int DT, int XT>
__global__ void __launch_bounds__(1024)
k_norm_bwd_dx(NormBwdArgs a) {
  constexpr int V = 4;
  __shared__ f2_t part[2][16];
  const int64_t row = blockIdx.x;
  const float mu = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
  Raw8<DT> y[V];
  Raw8<XT> x[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t col = (int64_t)(v * 1024 + threadIdx.x) * 8;
    y[v] = load_raw8<DT, false>(a.dy, row, col, a.K);
    x[v] = load_raw8<XT, false, true>(a.x, row, col, a.K);
  }
  float st = 0.f, sx = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float d[8], h[8], g[8];
    params8<false>(a.gamma, a.pdt, (int64_t)(v * 1024 + threadIdx.x) * 8, a.K, 1.f, g);
    values8<DT>(y[v], d);
    xhat8<XT>(x[v], mu, rstd, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float tt = d[e] * g[e];
      st += tt;
      sx = fmaf(tt, h[e], sx);
    }
  }
  const f2_t sums = row_sums<1024>(st, sx, part, 0);
  const float mt = a.mean ? sums[0] / (float)a.K : 0.f, mx = sums[1] / (float)a.K;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t col = (int64_t)(v * 1024 + threadIdx.x) * 8;
    float d[8], h[8], g[8];
    params8<false>(a.gamma, a.pdt, col, a.K, 1.f, g);
    values8<DT>(y[v], d);
    xhat8<XT>(x[v], mu, rstd, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = rstd * fmaf(-mx, h[e], fmaf(d[e], g[e], -mt));
    store_row8<DT, false>(a.dx, nullptr, row, a.lddx, col, a.K, d);
  }
}

// Longer rows, first kernel: the column sums of rows blockIdx.y, blockIdx.y + gridDim.y, ...; 8 columns a thread.
template <int DT, int XT>
__global__ void __launch_bounds__(256)
k_norm_bwd_long_cols(NormBwdArgs a) {
  const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= a.K) return;
  float dg[8], db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dg[e] = db[e] = 0.f;
  for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y) {
    const float mu = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
    float d[8], h[8];
    values8<DT>(load_raw8<DT, true>(a.dy, row, col, a.K), d);
    values8<XT>(load_raw8<XT, true>(a.x, row, col, a.K), h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dg[e] = fmaf(d[e], (h[e] - mu) * rstd, dg[e]);
      db[e] += d[e];
    }
  }
  float* const og = gridDim.y == 1 ? a.dgamma : a.part + (int64_t)blockIdx.y * 2 * a.K;
  float* const ob = gridDim.y == 1 ? a.dbeta : a.part + ((int64_t)blockIdx.y * 2 + 1) * a.K;
  if (og) store8<2>(og, col, a.K - col, dg);
  if (ob) store8<2>(ob, col, a.K - col, db);
}

// dgamma and dbeta from the blocks' column sums: 64 columns a block, 16 threads a column that each add every 16th block's
// in turn, joined in a fixed order. No blocks (no rows): zeros.
__global__ void __launch_bounds__(1024)
k_norm_cols(const float* __restrict__ part, int blocks, int64_t K, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float s[16][64];
  const int c = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + c;     // column of [dgamma | dbeta]
  float v = 0.f;
  if (i < 2 * K) {
    const float* p = part + i;
    int b = w;
    for (; b + 112 < blocks; b += 128) {         // eight loads in flight
      float t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = p[(int64_t)(b + 16 * j) * 2 * K];
#pragma unroll
      for (int j = 0; j < 8; ++j) v += t[j];
    }
    for (; b < blocks; b += 16) v += p[(int64_t)b * 2 * K];
  }
  s[w][c] = v;
  __syncthreads();
  if (w || i >= 2 * K) return;
#pragma unroll
  for (int j = 1; j < 16; ++j) v += s[j][c];
  if (i < K) {
    if (dgamma) dgamma[i] = v;
  } else if (dbeta) {
    dbeta[i - K] = v;
  }
}

// ------------------------------------------------------------------------------------- host
bool float_type(int dt) { return dt == SLIM_F16 || dt == SLIM_BF16 || dt == SLIM_F32; }
size_t elem(int dt) { return dt == SLIM_F32 ? 4 : 2; }

// Rows past 16384, and in the backward fp32 rows past 8192 that end inside a vector, may take a block of 1024 threads each, and a
// launch holds fewer than 2^32 threads.
constexpr int64_t kMostLong = int64_t(1) << 22;
bool too_many(int64_t M, int64_t K) { return K > 16384 && M >= kMostLong; }
bool too_many_bwd(int64_t M, int64_t K, int dtype) { return dtype == SLIM_F32 && K > 8192 && K % 8 && M >= kMostLong; }

template <int DT, int YT, bool RAG>
void norm_rows(const NormArgs& a, SlimKernelTimer& timer, hipStream_t s) {
  const auto grid = [&](int64_t units, int64_t most) { return dim3((unsigned)(units < most ? units : most)); };
  if (a.K <= 512) SLIM_LAUNCH(timer, (k_norm<DT, YT, 64, 1, true, true, RAG>), grid((a.M + 3) / 4, 2048), dim3(256), s, a);
  else if (a.K <= 1024) SLIM_LAUNCH(timer, (k_norm<DT, YT, 64, 2, true, true, RAG>), grid((a.M + 3) / 4, 2048), dim3(256), s, a);
  else if (a.K <= 4096) SLIM_LAUNCH(timer, (k_norm<DT, YT, 256, 2, true, true, RAG>), grid(a.M, 1024), dim3(256), s, a);
  else if (a.K <= 8192) SLIM_LAUNCH(timer, (k_norm<DT, YT, 512, 2, true, true, RAG>), grid(a.M, 512), dim3(512), s, a);
  else if (a.K <= 16384) SLIM_LAUNCH(timer, (k_norm<DT, YT, 512, 4, true, true, RAG>), grid(a.M, 512), dim3(512), s, a);
  else if (!RAG && a.K <= 32768) SLIM_LAUNCH(timer, (k_norm<DT, YT, 512, 8, false, false, false>), grid(a.M, 512), dim3(512), s, a);
  else SLIM_LAUNCH(timer, (k_norm_long<DT, YT>), dim3((unsigned)a.M), dim3(1024), s, a);
}

template <int DT>
void norm_to(const NormArgs& a, int ydt, SlimKernelTimer& timer, hipStream_t s) {
  const bool rag = a.K % 8 != 0;
  if (ydt == SLIM_Q8_E4M3) rag ? norm_rows<DT, kQ8, true>(a, timer, s) : norm_rows<DT, kQ8, false>(a, timer, s);
  else rag ? norm_rows<DT, DT, true>(a, timer, s) : norm_rows<DT, DT, false>(a, timer, s);
}

// Blocks of the backward, each with a row of column sums that a second launch adds; up to four rounds of one block are
// less than that launch takes. Long rows: about 1024 blocks of column sums, 2048 columns wide (2048 x 28672 in bf16, sums and
// their joining: 512 blocks 48 us, 1024 47, 2048 54, 4096 67), of at least four rows each, so that sums are not all that is
// written (111 x 19715: column sums 9.7 us, with a block a row 18.2).
int64_t bwd_blocks(int64_t M, int64_t K) {
  if (K > 16384) return std::max<int64_t>(1, std::min(M / 4, 1024 / ((K + 2047) / 2048)));
  const int64_t units = K <= 1024 ? (M + 3) / 4 : M, most = K <= 4096 ? 768 : K <= 8192 ? 512 : 256;
  return units <= 4 ? 1 : units < most ? units : most;
}

template <int DT, int XT, bool RAG>
void norm_bwd_rows_of(const NormBwdArgs& a, hipStream_t s) {
  const unsigned blocks = (unsigned)bwd_blocks(a.M, a.K);
  SlimKernelTimer timer("norm_bwd", s);
  if (a.K <= 512) SLIM_LAUNCH(timer, (k_norm_bwd<DT, XT, 64, 1, true, true, RAG>), dim3(blocks), dim3(256), s, a);
  else if (a.K <= 1024) SLIM_LAUNCH(timer, (k_norm_bwd<DT, XT, 64, 2, true, true, RAG>), dim3(blocks), dim3(256), s, a);
  else if (a.K <= 4096) SLIM_LAUNCH(timer, (k_norm_bwd<DT, XT, 256, 2, true, true, RAG>), dim3(blocks), dim3(256), s, a);
  else if (a.K <= 8192) SLIM_LAUNCH(timer, (k_norm_bwd<DT, XT, 256, 4, true, true, RAG>), dim3(blocks), dim3(256), s, a);
  // (8-bit rows that end inside a vector without the next row ahead, which would spill: 2000 x 12287 44 us, 53 with it)
  else if (a.K <= 16384 && !(RAG && DT == 2))
    SLIM_LAUNCH(timer, (k_norm_bwd<DT, XT, 512, 4, DT != 2, DT != 2 && !(RAG && XT == kQ8), RAG && DT != 2>), dim3(blocks), dim3(512), s, a);
  else {
    // the column sums first: dX may be written over dY
    SLIM_LAUNCH(timer, (k_norm_bwd_long_cols<DT, XT>), dim3((unsigned)((a.K + 2047) / 2048), blocks), dim3(256), s, a);
    SlimKernelTimer timer2("norm_bwd_dx", s);
    if (!RAG && a.K <= 32768) SLIM_LAUNCH(timer2, (k_norm_bwd_dx<DT, XT>), dim3((unsigned)a.M), dim3(1024), s, a);
    else SLIM_LAUNCH(timer2, (k_norm_bwd_long<DT, XT>), dim3((unsigned)a.M), dim3(1024), s, a);
  }
}

template <int DT, int XT>
void norm_bwd_rows(const NormBwdArgs& a, hipStream_t s) {
  a.K % 8 ? norm_bwd_rows_of<DT, XT, true>(a, s) : norm_bwd_rows_of<DT, XT, false>(a, s);
}

}  // namespace

extern "C" int slim_norm(const void* X, int dtype, int64_t M, int64_t K, int64_t ldx, const void* gamma, const void* beta,
                         int pdtype, int rms, float eps, void* Y, int ydtype, int64_t ldy, uint8_t* yexps, float* mean,
                         float* rstd, void* stream) {
  if (!float_type(dtype) || !float_type(pdtype) || (ydtype != dtype && ydtype != SLIM_Q8_E4M3)) return SLIM_EDTYPE;
  const bool q8 = ydtype == SLIM_Q8_E4M3;
  if (M < 0 || K < 1 || K > kMaxRow8 || M > 0x7FFFFFFF || ldx < K || (!q8 && ldy < K)) return SLIM_ESHAPE;
  if (!(eps >= 0.f) || (rms && beta)) return SLIM_EINVAL;
  if (too_many(M, K)) return SLIM_EUNSUPPORTED;
  if (M == 0) return SLIM_OK;
  if (!X || !Y || !rstd || (q8 && !yexps)) return SLIM_EINVAL;
  if (!slim_aligned_to(X, elem(dtype)) || !slim_aligned_to(Y, q8 ? 16 : elem(dtype)) || !slim_aligned16(yexps) ||
      !slim_aligned_to(gamma, elem(pdtype)) || !slim_aligned_to(beta, elem(pdtype)) || !slim_aligned_to(mean, 4) ||
      !slim_aligned_to(rstd, 4))
    return SLIM_EALIGN;
  const NormArgs a{{X, nullptr, ldx}, gamma, beta, pdtype, rms != 0, eps, M, K, Y, ldy, yexps, mean, rstd};
  hipStream_t s = (hipStream_t)stream;
  SlimKernelTimer timer("norm", s);
  if (dtype == SLIM_F16) norm_to<0>(a, ydtype, timer, s);
  else if (dtype == SLIM_BF16) norm_to<1>(a, ydtype, timer, s);
  else norm_to<2>(a, ydtype, timer, s);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

extern "C" int slim_norm_bwd_workspace(int64_t M, int64_t K, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  if (M < 0 || K < 1 || K > kMaxRow8 || M > 0x7FFFFFFF) return SLIM_ESHAPE;
  if (too_many(M, K)) return SLIM_EUNSUPPORTED;
  const int64_t blocks = M > 0 ? bwd_blocks(M, K) : 0;
  *bytes = blocks > 1 ? (size_t)blocks * 2 * (size_t)K * 4 : 0;
  return SLIM_OK;
}

extern "C" int slim_norm_bwd(const void* dY, int dtype, int64_t lddy, const void* X, int xdtype, const uint8_t* xexps,
                             int64_t ldx, int64_t M, int64_t K, const void* gamma, int pdtype, const float* mean,
                             const float* rstd, void* dX, int64_t lddx, float* dgamma, float* dbeta, void* ws,
                             size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = slim_norm_bwd_workspace(M, K, &need);
  if (rc != SLIM_OK) return rc;
  const bool q8 = xdtype == SLIM_Q8_E4M3;
  if (!float_type(dtype) || !float_type(pdtype) || (xdtype != dtype && !q8)) return SLIM_EDTYPE;
  if (lddy < K || (!q8 && ldx < K) || lddx < K) return SLIM_ESHAPE;
  if (too_many_bwd(M, K, dtype)) return SLIM_EUNSUPPORTED;
  if (M > 0 && (!dY || !X || !rstd || !dX || (q8 && !xexps))) return SLIM_EINVAL;
  if (!slim_aligned_to(dY, elem(dtype)) || !slim_aligned_to(X, q8 ? 16 : elem(dtype)) || !slim_aligned16(xexps) ||
      !slim_aligned_to(gamma, elem(pdtype)) || !slim_aligned_to(mean, 4) || !slim_aligned_to(rstd, 4) ||
      !slim_aligned_to(dX, elem(dtype)) || !slim_aligned_to(dgamma, 4) || !slim_aligned_to(dbeta, 4))
    return SLIM_EALIGN;
  if (need && (!ws || ws_bytes < need)) return SLIM_EWORKSPACE;
  if (need && !slim_aligned16(ws)) return SLIM_EALIGN;
  hipStream_t s = (hipStream_t)stream;
  const NormBwdArgs a{{dY, nullptr, lddy}, {X, xexps, q8 ? q8_row(K) : ldx}, gamma, pdtype, mean, rstd, M, K, dX, lddx,
                      reinterpret_cast<float*>(ws), dgamma, dbeta};
  if (M > 0) {
    if (dtype == SLIM_F16) q8 ? norm_bwd_rows<0, kQ8>(a, s) : norm_bwd_rows<0, 0>(a, s);
    else if (dtype == SLIM_BF16) q8 ? norm_bwd_rows<1, kQ8>(a, s) : norm_bwd_rows<1, 1>(a, s);
    else q8 ? norm_bwd_rows<2, kQ8>(a, s) : norm_bwd_rows<2, 2>(a, s);
    if (hipGetLastError() != hipSuccess) return SLIM_EDEVICE;
  }
  if ((dgamma || dbeta) && (M == 0 || bwd_blocks(M, K) > 1)) {
    SlimKernelTimer timer("norm_cols", s);
    SLIM_LAUNCH(timer, k_norm_cols, dim3((unsigned)((2 * K + 63) / 64)), dim3(1024), s, reinterpret_cast<const float*>(ws),
                (int)(M > 0 ? bwd_blocks(M, K) : 0), K, dgamma, dbeta);
  }
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
