// grad_w8.hip - the weight gradient from an 8-bit checkpoint of the activations: slim_grad_w8.
//
// D[k][n] = sum_m X[m][k] dY[m][n] (= grad W^T). The reduction runs along the stored rows of both operands, so a power of
// two for each row and group cannot be taken out of the sum: the codes are widened to dY's 16-bit type with their exponent
// on the way into LDS (exact in bf16, and in fp16 for checkpoints of fp16 values below 63488), and the products run on
// v_mfma_f32_32x32x16 with fp32 accumulators. X moves at half the bytes of a 16-bit activation.
#include <hip/hip_runtime.h>

#include "slim_launch.h"
#include "slim_q8.h"
#include "slim_timing.h"

typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef short s4_t __attribute__((ext_vector_type(4)));

namespace {

constexpr int kWM = 32;       // rows of one chunk of the reduction

template <int DT>
SLIM_DEV f16_t mfma_acc(u32x2_t a0, u32x2_t a1, u32x2_t b0, u32x2_t b1, f16_t c) {
  const u32x4_t a = {a0[0], a0[1], a1[0], a1[1]}, b = {b0[0], b0[1], b1[0], b1[1]};
  if constexpr (DT == 1)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, a), __builtin_bit_cast(bf8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8_t, a), __builtin_bit_cast(h8_t, b), c, 0, 0, 0);
}

// Four 16-bit values at `p` (LDS) for lane 16 G + 4 a + b: element b of the 8-byte rows that lanes 16 G + a + 4 i address.
SLIM_DEV u32x2_t read_tr(const uint8_t* p) {
  typedef __attribute__((address_space(3))) s4_t* lds_s4;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(void*)p));
}

// Byte offset of 16-bit column c of row r in 256-byte LDS rows; the 32-byte pieces are XOR-swizzled by 2 (row % 4), so that
// the four rows that one group of 16 lanes reads at once fall in distinct banks.
SLIM_DEV uint32_t lds_at(int r, int c) {
  return (uint32_t)r * 256u + ((uint32_t)((c >> 4) ^ (2 * (r & 3))) << 5) + (uint32_t)((c & 15) * 2);
}

// Four consecutive positions k .. k + 3 of row n of the gradient: all of them, or the two that the pattern keeps.
SLIM_DEV void store_grad4(float* gW, const uint8_t* meta, int64_t n, int64_t k, int64_t K, f4_t v) {
  if (meta) {
    const uint32_t nib = (uint32_t)(meta[n * (K / 8) + k / 8] >> (k & 4)) & 0xFu;
    const uint32_t i0 = nib & 3u, i1 = nib >> 2;
    const f2_t o = {i0 == 0 ? v[0] : i0 == 1 ? v[1] : i0 == 2 ? v[2] : v[3], i1 == 0 ? v[0] : i1 == 1 ? v[1] : i1 == 2 ? v[2] : v[3]};
    *reinterpret_cast<f2_t*>(gW + n * (K / 2) + k / 2) = o;
  } else if (k + 4 <= K) {
    __builtin_memcpy(gW + n * K + k, &v, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k + e < K) gW[n * K + k + e] = v[e];
  }
}

// 128 (k) x 128 (n) tiles, four waves of 64 x 64; chunks of 32 rows through registers into two LDS slots.
template <int DT>
__global__ void __launch_bounds__(256)
k_wgrad8(const uint16_t* __restrict__ dY, int64_t lddy, const uint8_t* __restrict__ xc, const uint8_t* __restrict__ xe, int64_t M,
         int64_t N, int64_t K, const uint8_t* __restrict__ meta, float* __restrict__ gW) {
  __shared__ __attribute__((aligned(16))) uint8_t lx[2][kWM * 256], ly[2][kWM * 256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t Kp = q8_row(K), Ge = q8_exp_row(K), tk = Kp / 128;
  const int64_t n0 = (int64_t)(blockIdx.x / tk) * 128, k0 = (int64_t)(blockIdx.x % tk) * 128;
  // staging: row tid / 8 of the chunk, columns 16 (tid % 8) .. + 15
  const int row = tid >> 3, col = 16 * (tid & 7);
  const int64_t nleft = N - n0 - col;
  u32x4_t y0, y1, c;
  float sc;
  auto load = [&](int64_t m) {
    m += row;
    y0 = y1 = c = u32x4_t{0, 0, 0, 0};
    sc = 0.f;
    if (m >= M) return;
    const uint16_t* p = dY + m * lddy + n0 + col;
    if (nleft >= 16) {
      __builtin_memcpy(&y0, p, 16);
      __builtin_memcpy(&y1, p + 8, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y0[e] = (2 * e < nleft ? (uint32_t)p[2 * e] : 0u) | (2 * e + 1 < nleft ? (uint32_t)p[2 * e + 1] << 16 : 0u);
        y1[e] = (2 * e + 8 < nleft ? (uint32_t)p[2 * e + 8] : 0u) | (2 * e + 9 < nleft ? (uint32_t)p[2 * e + 9] << 16 : 0u);
      }
    }
    c = *reinterpret_cast<const u32x4_t*>(xc + m * Kp + k0 + col);
    sc = q8_pow2(xe[m * Ge + k0 / 128]);
  };
  auto put = [&](int z) {
    uint8_t* y = &ly[z][lds_at(row, col)];
    *reinterpret_cast<u32x4_t*>(y) = y0;
    *reinterpret_cast<u32x4_t*>(y + 16) = y1;
    u32x4_t v[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f[4];
      q8_values4(c[e], sc, f);
      v[e >> 1][2 * (e & 1)] = to_16<DT>(f[0]) | to_16<DT>(f[1]) << 16;
      v[e >> 1][2 * (e & 1) + 1] = to_16<DT>(f[2]) | to_16<DT>(f[3]) << 16;
    }
    uint8_t* x = &lx[z][lds_at(row, col)];
    *reinterpret_cast<u32x4_t*>(x) = v[0];
    *reinterpret_cast<u32x4_t*>(x + 16) = v[1];
  };
  f16_t acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i >> 1][i & 1][e] = 0.f;
  const int G = lane >> 4, q = lane & 15, wk = 64 * (wave & 1), wn = 64 * (wave >> 1);
  const int rr = 8 * (G >> 1) + (q >> 2), cr = 16 * (G & 1) + 4 * (q & 3);
  load(0);
  put(0);
  __syncthreads();
  int z = 0;
  for (int64_t m = 0; m < M; m += kWM, z ^= 1) {
    const bool more = m + kWM < M;
    if (more) load(m + kWM);
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      u32x2_t a[2][2], b[2][2];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          a[f][j] = read_tr(&lx[z][lds_at(16 * st + rr + 4 * j, wk + 32 * f + cr)]);
          b[f][j] = read_tr(&ly[z][lds_at(16 * st + rr + 4 * j, wn + 32 * f + cr)]);
        }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) acc[x][y] = mfma_acc<DT>(a[x][0], a[x][1], b[y][0], b[y][1], acc[x][y]);
    }
    if (more) put(z ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int64_t n = n0 + wn + 32 * y + (lane & 31);
    if (n >= N) continue;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t k = k0 + wk + 32 * x + 8 * i + 4 * (lane >> 5);
        if (k < K)
          store_grad4(gW, meta, n, k, K, f4_t{acc[x][y][4 * i], acc[x][y][4 * i + 1], acc[x][y][4 * i + 2], acc[x][y][4 * i + 3]});
      }
  }
}

}  // namespace

extern "C" int slim_grad_w8(const void* dY, int dtype, int64_t lddy, const uint8_t* xcodes, const uint8_t* xexps, int64_t M,
                            int64_t N, int64_t K, const uint8_t* meta, float* gW, void* stream) {
  if (dtype != SLIM_F16 && dtype != SLIM_BF16) return SLIM_EDTYPE;
  if (M < 0 || N < 1 || K < 1 || N > kMaxRow8 || K > kMaxRow8 || lddy < N || (meta && K % 16)) return SLIM_ESHAPE;
  if (!gW || (M > 0 && (!dY || !xcodes || !xexps))) return SLIM_EINVAL;
  if (!slim_aligned_to(dY, 2) || !slim_aligned16(xcodes) || !slim_aligned16(xexps) || !slim_aligned16(meta) ||
      !slim_aligned16(gW))
    return SLIM_EALIGN;
  const int64_t tiles = ((N + 127) / 128) * ((K + 127) / 128);
  if (tiles > 0x7FFFFFFF) return SLIM_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  SlimKernelTimer timer("grad_w8", s);
  if (dtype == SLIM_F16)
    SLIM_LAUNCH(timer, k_wgrad8<0>, dim3((unsigned)tiles), dim3(256), s, reinterpret_cast<const uint16_t*>(dY), lddy, xcodes,
                xexps, M, N, K, meta, gW);
  else
    SLIM_LAUNCH(timer, k_wgrad8<1>, dim3((unsigned)tiles), dim3(256), s, reinterpret_cast<const uint16_t*>(dY), lddy, xcodes,
                xexps, M, N, K, meta, gW);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
