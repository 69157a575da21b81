// act8.hip - activations and weights in 8 bits: slim_quant8, slim_dequant8, slim_pack8.
#include <hip/hip_runtime.h>

#include "slim_launch.h"
#include "slim_q8.h"
#include "slim_timing.h"

namespace {

// --------------------------------------------------------------------------- activations
// One group of 128 consecutive values of a row per 8 lanes, 16 values a lane: the group's largest magnitude over the
// eight lanes, its exponent, and 16 codes a lane in one 16-byte store. Groups are numbered row by row, so the lanes of a
// wave read eight groups that follow each other. Bound by HBM (2 or 4 bytes in, 1 + 1/128 out per value). A launch by itself, X
// from memory: 8192 x 8192 in bf16 36.5 us (5.5 TB/s), 8192 x 28672 127 us (5.6 TB/s), in fp32 8192 x 8192 57.8 us (5.8 TB/s);
// 1 x 4096 5.5 us, 2.0 as one of many in a graph.
template <int DT>
__global__ void __launch_bounds__(256)
k_quant8(const void* __restrict__ X, int64_t ldx, uint32_t K, uint32_t G, uint32_t total, uint8_t* __restrict__ codes,
         uint8_t* __restrict__ exps) {
  const uint32_t u = blockIdx.x * 32 + (threadIdx.x >> 3), sub = threadIdx.x & 7;
  if (u >= total) return;      // whole groups of 8 lanes
  const uint32_t row = u / G, g = u - row * G, col = g * 128 + sub * 16;
  const int64_t left = (int64_t)K - col, at = (int64_t)row * ldx + col;
  float f[16];
  load8<DT>(X, at, left, f);
  load8<DT>(X, at + 8, left - 8, f + 8);
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) m = max(m, q8_abs(f[e]));
  const uint32_t b = q8_exponent(oct_max_u32(m));
  const float s = q8_inverse(b);
  u32x4_t c;
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = q8_codes4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3], s);
  *reinterpret_cast<u32x4_t*>(codes + ((int64_t)row * G + g) * 128 + sub * 16) = c;
  const uint32_t Ge = (G + 3) & ~3u;
  if (sub == 0) exps[(int64_t)row * Ge + g] = (uint8_t)b;
  else if (g == G - 1 && g + sub < Ge) exps[(int64_t)row * Ge + g + sub] = 0;   // the row's last word ends in zeros
}

// The values codes stand for, 16 a lane, in the order of k_quant8; every one below 2^128 is exact in fp32, and in bf16 from 2^-130
// on (multiples of 2^-135 at e = -126). A launch by itself, codes from memory: 8192 x 8192 to bf16 34.4 us (5.9 TB/s), 8192 x 28672
// 124 us, to fp32 8192 x 8192 75.9 us (4.4 TB/s; 16 values a lane side by side, 64 bytes, 99.9).
template <int DT>
__global__ void __launch_bounds__(256)
k_dequant8(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps, uint32_t K, uint32_t G, uint32_t total,
           void* __restrict__ Y, int64_t ldy) {
  const uint32_t u = blockIdx.x * 32 + (threadIdx.x >> 3), sub = threadIdx.x & 7;
  if (u >= total) return;
  const uint32_t row = u / G, g = u - row * G, col = g * 128 + sub * 16;
  const float s = q8_pow2(exps[(int64_t)row * ((G + 3) & ~3u) + g]);
  if constexpr (DT == 2) {
    // eight lanes write 128 bytes together, four times
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t at = 32 * e + 4 * sub;
      float f[4];
      q8_values4(*reinterpret_cast<const uint32_t*>(codes + ((int64_t)row * G + g) * 128 + at), s, f);
      const int64_t k = g * 128 + at;
      float* y = reinterpret_cast<float*>(Y) + (int64_t)row * ldy + k;
      if (k + 4 <= K) {
        __builtin_memcpy(y, f, 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k + i < K) y[i] = f[i];
      }
    }
    return;
  }
  const u32x4_t c = *reinterpret_cast<const u32x4_t*>(codes + ((int64_t)row * G + g) * 128 + sub * 16);
  float f[16];
#pragma unroll
  for (int e = 0; e < 4; ++e) q8_values4(c[e], s, f + 4 * e);
  const int64_t left = (int64_t)K - col, at = (int64_t)row * ldy + col;
  store8<DT>(Y, at, left, f);
  store8<DT>(Y, at + 8, left - 8, f + 8);
}

// --------------------------------------------------------------------------- weights
// One 128 x 128 block of W per workgroup: its largest magnitude, its exponent, and its codes as tiles of 16 rows x 128
// reduction positions (see include/slim.h). Codes go through LDS row by row; the same LDS image read by columns gives
// the transposed pack, whose blocks have the same exponents. Once a step at most: 28672 x 8192 from fp32 240 us, with both packs
// 271 us (5.2 TB/s).
// Piece i of 1024: 16 codes, row i / 8, columns 16 (i % 8) ..
template <int DT>
__global__ void __launch_bounds__(256)
k_pack8(const void* __restrict__ W, int64_t ldw, int64_t N, int64_t K, uint8_t* __restrict__ codes, uint8_t* __restrict__ exps,
        uint8_t* __restrict__ codesT, uint8_t* __restrict__ expsT) {
  __shared__ __attribute__((aligned(16))) uint8_t img[128 * 144];
  __shared__ uint32_t part[4];
  const int tid = threadIdx.x;
  const int64_t nb = blockIdx.x, kb = blockIdx.y, n0 = nb * 128, k0 = kb * 128;
  float f[4][16];
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = tid + 256 * j;
    const int64_t n = n0 + (i >> 3), k = k0 + 16 * (i & 7);
    const int64_t left = n < N ? K - k : 0;
    load8<DT>(W, n * ldw + k, left, f[j]);
    load8<DT>(W, n * ldw + k + 8, left - 8, f[j] + 8);
#pragma unroll
    for (int e = 0; e < 16; ++e) m = max(m, q8_abs(f[j][e]));
  }
  m = wave_max_u32(m);
  if ((tid & 63) == 0) part[tid >> 6] = m;
  __syncthreads();
  const uint32_t b = q8_exponent(max(max(part[0], part[1]), max(part[2], part[3])));
  const float s = q8_inverse(b);
  const int64_t G = (K + 127) / 128, GT = (N + 127) / 128, Nt = (N + 15) / 16, Kt = (K + 15) / 16;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = tid + 256 * j;
    u32x4_t c;
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = q8_codes4(f[j][4 * e], f[j][4 * e + 1], f[j][4 * e + 2], f[j][4 * e + 3], s);
    *reinterpret_cast<u32x4_t*>(&img[(i >> 3) * 144 + 16 * (i & 7)]) = c;
  }
  __syncthreads();
  // piece p of a tile: half p / 64, column block (p / 16) % 4, row p % 16
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = tid + 256 * j, t = i >> 7, p = i & 127, row = 16 * t + (p & 15), col = 32 * ((p >> 4) & 3) + 16 * (p >> 6);
    if (codes && n0 / 16 + t < Nt)
      *reinterpret_cast<u32x4_t*>(codes + ((n0 / 16 + t) * G + kb) * 2048 + 16 * p) =
          *reinterpret_cast<const u32x4_t*>(&img[row * 144 + col]);
    if (codesT && k0 / 16 + t < Kt) {
      u32x4_t c;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c[e] = (uint32_t)img[(col + 4 * e) * 144 + row] | (uint32_t)img[(col + 4 * e + 1) * 144 + row] << 8 |
               (uint32_t)img[(col + 4 * e + 2) * 144 + row] << 16 | (uint32_t)img[(col + 4 * e + 3) * 144 + row] << 24;
      *reinterpret_cast<u32x4_t*>(codesT + ((k0 / 16 + t) * GT + nb) * 2048 + 16 * p) = c;
    }
  }
  const int64_t Ge = q8_exp_row(K), GTe = q8_exp_row(N);
  if (tid == 0 && codes) exps[nb * Ge + kb] = (uint8_t)b;
  if (tid == 1 && codesT) expsT[kb * GTe + nb] = (uint8_t)b;
  // the words that end a row of exponents end in zeros
  if (tid >= 4 && tid < 8 && codes && kb == G - 1 && kb + tid - 3 < Ge) exps[nb * Ge + kb + tid - 3] = 0;
  if (tid >= 8 && tid < 12 && codesT && nb == GT - 1 && nb + tid - 7 < GTe) expsT[kb * GTe + nb + tid - 7] = 0;
}

}  // namespace

extern "C" int slim_quant8(const void* X, int dtype, int64_t M, int64_t K, int64_t ldx, uint8_t* codes, uint8_t* exps,
                           void* stream) {
  if (M < 0 || K < 1 || K > kMaxRow8 || ldx < K) return SLIM_ESHAPE;
  if (dtype != SLIM_F16 && dtype != SLIM_BF16 && dtype != SLIM_F32) return SLIM_EDTYPE;
  if (M == 0) return SLIM_OK;
  if (!X || !codes || !exps) return SLIM_EINVAL;
  if (!slim_aligned_to(X, dtype == SLIM_F32 ? 4 : 2) || !slim_aligned16(codes) || !slim_aligned16(exps)) return SLIM_EALIGN;
  const int64_t G = (K + 127) / 128;
  if (M > kMaxQuant8 / G) return SLIM_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  const uint32_t total = (uint32_t)(M * G);
  const dim3 grid((unsigned)((M * G + 31) / 32));
  SlimKernelTimer timer("quant8", s);
  if (dtype == SLIM_F16)
    SLIM_LAUNCH(timer, k_quant8<0>, grid, dim3(256), s, X, ldx, (uint32_t)K, (uint32_t)G, total, codes, exps);
  else if (dtype == SLIM_BF16)
    SLIM_LAUNCH(timer, k_quant8<1>, grid, dim3(256), s, X, ldx, (uint32_t)K, (uint32_t)G, total, codes, exps);
  else
    SLIM_LAUNCH(timer, k_quant8<2>, grid, dim3(256), s, X, ldx, (uint32_t)K, (uint32_t)G, total, codes, exps);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

extern "C" int slim_dequant8(const uint8_t* codes, const uint8_t* exps, int64_t M, int64_t K, void* Y, int dtype, int64_t ldy,
                             void* stream) {
  if (M < 0 || K < 1 || K > kMaxRow8 || ldy < K) return SLIM_ESHAPE;
  if (dtype != SLIM_F16 && dtype != SLIM_BF16 && dtype != SLIM_F32) return SLIM_EDTYPE;
  if (M == 0) return SLIM_OK;
  if (!codes || !exps || !Y) return SLIM_EINVAL;
  if (!slim_aligned_to(Y, dtype == SLIM_F32 ? 4 : 2) || !slim_aligned16(codes) || !slim_aligned16(exps)) return SLIM_EALIGN;
  const int64_t G = (K + 127) / 128;
  if (M > kMaxQuant8 / G) return SLIM_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  const uint32_t total = (uint32_t)(M * G);
  const dim3 grid((unsigned)((M * G + 31) / 32));
  SlimKernelTimer timer("dequant8", s);
  if (dtype == SLIM_F16)
    SLIM_LAUNCH(timer, k_dequant8<0>, grid, dim3(256), s, codes, exps, (uint32_t)K, (uint32_t)G, total, Y, ldy);
  else if (dtype == SLIM_BF16)
    SLIM_LAUNCH(timer, k_dequant8<1>, grid, dim3(256), s, codes, exps, (uint32_t)K, (uint32_t)G, total, Y, ldy);
  else
    SLIM_LAUNCH(timer, k_dequant8<2>, grid, dim3(256), s, codes, exps, (uint32_t)K, (uint32_t)G, total, Y, ldy);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

extern "C" int slim_pack8(const void* W, int dtype, int64_t N, int64_t K, int64_t ldw, uint8_t* codes, uint8_t* exps,
                          uint8_t* codesT, uint8_t* expsT, void* stream) {
  if (N < 1 || K < 1 || N > kMaxRow8 || K > kMaxRow8 || ldw < K) return SLIM_ESHAPE;
  if (dtype != SLIM_F16 && dtype != SLIM_BF16 && dtype != SLIM_F32) return SLIM_EDTYPE;
  if (!W || (!codes && !codesT) || !codes != !exps || !codesT != !expsT) return SLIM_EINVAL;
  if (!slim_aligned_to(W, dtype == SLIM_F32 ? 4 : 2) || !slim_aligned16(codes) || !slim_aligned16(exps) ||
      !slim_aligned16(codesT) || !slim_aligned16(expsT))
    return SLIM_EALIGN;
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)((N + 127) / 128), (unsigned)((K + 127) / 128));
  SlimKernelTimer timer("pack8", s);
  if (dtype == SLIM_F16)
    SLIM_LAUNCH(timer, k_pack8<0>, grid, dim3(256), s, W, ldw, N, K, codes, exps, codesT, expsT);
  else if (dtype == SLIM_BF16)
    SLIM_LAUNCH(timer, k_pack8<1>, grid, dim3(256), s, W, ldw, N, K, codes, exps, codesT, expsT);
  else
    SLIM_LAUNCH(timer, k_pack8<2>, grid, dim3(256), s, W, ldw, N, K, codes, exps, codesT, expsT);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
