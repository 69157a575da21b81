// linear8.hip - the 8-bit product with a scale for each block of 128: slim_linear8.
//
// Y[m][n] = sum_g 2^(ex[m][g] + ew[n/128][g]) sum_{k in group g} cx[m][k] cw[n][k], e4m3 codes c, on the scaled MFMA
// v_mfma_scale_f32_16x16x128_f8f6f4: its reduction of 128 is one group, and the two exponents go in as its scale
// operands, so scaling costs no arithmetic of its own. Lane l of an operand holds the 32 codes 32 (l / 16) .. of row
// l % 16, and the scale byte for them; D element i of lane l is row 4 (l / 16) + i of the first operand, row l % 16 of the
// second. The weight is the first operand, so a lane's four results are four consecutive columns of Y.
// Precision: products are exact and the accumulators are fp32; the unit's sum of the 128 products of one instruction is a
// little coarser than fp32 (1.5e-5 of the result's norm measured against 64 bits, at K 512 as at 8192). Y is rounded once
// to 16 bits, whose steps are 30 (fp16) to 250 times (bf16) as large.
#include <hip/hip_runtime.h>

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

// ------------------------------------------------------------------------------------- few rows
// One tile of 16 weight rows and up to 16 FM rows of X per block; its eight waves take the groups of the reduction in
// turn and add their sums through LDS in wave order. Nothing is shared within the reduction, so weight tiles (2 KiB of
// consecutive bytes) and X fragments go straight from memory to registers. Bound by the weight's bytes.
template <int FM, int DT>
__global__ void __launch_bounds__(512)
k_linear8_few(const uint8_t* __restrict__ X, const uint8_t* __restrict__ ex, const uint8_t* __restrict__ W,
              const uint8_t* __restrict__ ew, int64_t M, int64_t N, int64_t G, uint16_t* __restrict__ Y, int64_t ldy) {
  __shared__ f4_t part[8][FM][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4;
  const int64_t t = blockIdx.x, m0 = (int64_t)blockIdx.y * (16 * FM), Ge = (G + 3) & ~int64_t(3);
  const uint8_t* w = W + t * G * 2048 + lane * 16;
  const uint8_t* sw = ew + (t / 8) * Ge;
  const uint8_t* x[FM];
  const uint8_t* sx[FM];
#pragma unroll
  for (int f = 0; f < FM; ++f) {
    const int64_t m = m0 + 16 * f + r < M ? m0 + 16 * f + r : M - 1;    // rows past the last repeat it; not stored
    x[f] = X + m * G * 128 + 32 * q;
    sx[f] = ex + m * Ge;
  }
  f4_t acc[FM];
#pragma unroll
  for (int f = 0; f < FM; ++f) acc[f] = f4_t{0.f, 0.f, 0.f, 0.f};
  for (int64_t g = wave; g < G; g += 8) {
    const u32x4_t w0 = *reinterpret_cast<const u32x4_t*>(w + g * 2048), w1 = *reinterpret_cast<const u32x4_t*>(w + g * 2048 + 1024);
    const int s = sw[g];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
      const u32x4_t x0 = *reinterpret_cast<const u32x4_t*>(x[f] + g * 128), x1 = *reinterpret_cast<const u32x4_t*>(x[f] + g * 128 + 16);
      acc[f] = mfma8(cat8(w0, w1), cat8(x0, x1), acc[f], s, sx[f][g]);
    }
  }
#pragma unroll
  for (int f = 0; f < FM; ++f) part[wave][f][lane] = acc[f];
  __syncthreads();
  if (wave >= FM) return;
  f4_t v = part[0][wave][lane];
#pragma unroll
  for (int i = 1; i < 8; ++i) v += part[i][wave][lane];
  const int64_t m = m0 + 16 * wave + r, n = 16 * t + 4 * q;
  if (m < M && n < N) store4_16<DT>(Y, m * ldy + n, N - n, v);
}

template <int DT>
void launch(const uint8_t* X, const uint8_t* ex, const uint8_t* W, const uint8_t* ew, int64_t M, int64_t N, int64_t G,
            uint16_t* Y, int64_t ldy, hipStream_t s) {
  const unsigned nt = (unsigned)((N + 15) / 16);
  SlimKernelTimer timer("linear8_few", s);
  if (M <= 16)
    SLIM_LAUNCH(timer, (k_linear8_few<1, DT>), dim3(nt), dim3(512), s, X, ex, W, ew, M, N, G, Y, ldy);
  else if (M <= 32)
    SLIM_LAUNCH(timer, (k_linear8_few<2, DT>), dim3(nt), dim3(512), s, X, ex, W, ew, M, N, G, Y, ldy);
  else
    SLIM_LAUNCH(timer, (k_linear8_few<4, DT>), dim3(nt, (unsigned)((M + 63) / 64)), dim3(512), s, X, ex, W, ew, M, N, G,
                Y, ldy);
}

size_t round256(size_t x) { return (x + 255) & ~size_t(255); }
size_t code_bytes(int64_t M, int64_t K) { return round256((size_t)M * (size_t)q8_row(K)); }

int check_sizes(int xdtype, int64_t M, int64_t N, int64_t K) {
  if (xdtype != SLIM_F16 && xdtype != SLIM_BF16 && xdtype != SLIM_F32 && xdtype != SLIM_Q8_E4M3) return SLIM_EDTYPE;
  if (M < 0 || N < 1 || K < 1 || N > kMaxRow8 || K > kMaxRow8) return SLIM_ESHAPE;
  if (M > kMaxGroups8 / (q8_row(K) / 128) || M > kMaxGroups8 / 128) return SLIM_EUNSUPPORTED;
  return SLIM_OK;
}

}  // namespace

extern "C" int slim_linear8_workspace(int xdtype, int64_t M, int64_t N, int64_t K, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  const int rc = check_sizes(xdtype, M, N, K);
  if (rc != SLIM_OK) return rc;
  *bytes = xdtype == SLIM_Q8_E4M3 ? 0 : code_bytes(M, K) + round256((size_t)M * (size_t)q8_exp_row(K));
  return SLIM_OK;
}

extern "C" int slim_linear8(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t N, int64_t K, int64_t ldx,
                            const uint8_t* codes, const uint8_t* exps, void* Y, int ydtype, int64_t ldy, void* ws,
                            size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = slim_linear8_workspace(xdtype, M, N, K, &need);
  if (rc != SLIM_OK) return rc;
  if (ydtype != SLIM_F16 && ydtype != SLIM_BF16) return SLIM_EDTYPE;
  const bool packed = xdtype == SLIM_Q8_E4M3;
  if (ldy < N || (!packed && ldx < K)) return SLIM_ESHAPE;
  if (M == 0) return SLIM_OK;
  if (!X || (packed && !xexps) || !codes || !exps || !Y) return SLIM_EINVAL;
  if (!slim_aligned_to(X, packed ? 16 : xdtype == SLIM_F32 ? 4 : 2) || !slim_aligned16(xexps) || !slim_aligned16(codes) ||
      !slim_aligned16(exps) || !slim_aligned_to(Y, 2))
    return SLIM_EALIGN;
  if (need && (!ws || ws_bytes < need)) return SLIM_EWORKSPACE;
  if (need && !slim_aligned16(ws)) return SLIM_EALIGN;
  hipStream_t s = (hipStream_t)stream;
  const uint8_t* xc = reinterpret_cast<const uint8_t*>(X);
  const uint8_t* xe = xexps;
  if (!packed) {
    uint8_t* c = reinterpret_cast<uint8_t*>(ws);
    uint8_t* e = c + code_bytes(M, K);
    const int q = slim_quant8(X, xdtype, M, K, ldx, c, e, stream);
    if (q != SLIM_OK) return q;
    xc = c;
    xe = e;
  }
  const int64_t G = q8_row(K) / 128;
  if (ydtype == SLIM_F16) launch<0>(xc, xe, codes, exps, M, N, G, reinterpret_cast<uint16_t*>(Y), ldy, s);
  else launch<1>(xc, xe, codes, exps, M, N, G, reinterpret_cast<uint16_t*>(Y), ldy, s);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
