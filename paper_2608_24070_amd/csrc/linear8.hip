// linear8.hip - the 8-bit product with a scale for each block of 128: slim_linear8.
//
// Y[m][n] = sum_g 2^(ex[m][g] + ew[n/128][g]) sum_{k in group g} cx[m][k] cw[n][k], e4m3 codes c, on the scaled MFMA
// v_mfma_scale_f32_16x16x128_f8f6f4: its reduction of 128 is one group, and the two exponents go in as its scale
// operands, so scaling costs no arithmetic of its own. Lane l of an operand holds the 32 codes 32 (l / 16) .. of row
// l % 16, and the scale byte for them; D element i of lane l is row 4 (l / 16) + i of the first operand, row l % 16 of the
// second. The weight is the first operand, so a lane's four results are four consecutive columns of Y.
// Precision: the accumulators are fp32, but the unit adds the products of eight consecutive reduction positions (one lane's
// eight bytes) first, aligned to the largest of them and cut towards zero below 2^-13 of its leading bit (found with single
// pairs of products of known sizes; the unscaled fp8 instructions do the same); across the eights it keeps 24 bits. So each eight
// lose less than 7 2^-13 of their largest product. Against 64 bits that is 2e-5 of the result's norm for operands of one size
// throughout, and 4.5e-5 where a hundredth of X's channels is twenty times the rest; one sign in all operands leaves no bias that
// shows (below 1e-6). Y's rounding to 16 bits is 2.1e-4 (fp16) and 1.7e-3 (bf16) of its norm: with both, 45 x 13824 x 5120 in fp16 is
// 2.12e-4 from 64 bits where fp32 sums would be 2.07e-4, and one element in seven is the neighbouring fp16 value. The operands'
// own rounding to e4m3 is some hundred times as large. An fp32 Y would promise more than the unit holds, and is not offered; exact
// sums would take 16-bit products, at half the rate.
#include "linear8_product.h"

namespace {

template <int FM, int NT, int U, int XT, int DT>
__global__ void __launch_bounds__(512)
k_linear8_few(const uint8_t* __restrict__ X, const uint8_t* __restrict__ ex, int64_t ldx, int K, const uint8_t* __restrict__ W,
              const uint8_t* __restrict__ ew, int M, int64_t N, int G, uint16_t* __restrict__ Y, int64_t ldy) {
  few_body<FM, NT, U, XT>(X, ex, ldx, K, W, ew, M, N, G, StoreRows<DT>{Y, ldy});
}

template <int FM, int WN, int DT>
__global__ void __launch_bounds__(256, 1)
k_linear8_tile(const uint8_t* __restrict__ X, const uint8_t* __restrict__ ex, const uint8_t* __restrict__ W,
               const uint8_t* __restrict__ ew, int64_t M, int64_t N, int G, int fours, uint16_t* __restrict__ Y, int64_t ldy,
               float* __restrict__ sums) {
  tile_body<FM, WN>(X, ex, W, ew, M, N, G, fours, sums, [&] { return StoreRows<DT>{Y, ldy}; });
}

// The slices' sums in slice order, four columns a thread, `quads` of them a row.
template <int DT>
__global__ void __launch_bounds__(256)
k_linear8_sum(const f4_t* __restrict__ sums, int slices, uint32_t total, uint32_t quads, int64_t N, uint16_t* __restrict__ Y, int64_t ldy) {
  const uint32_t u = blockIdx.x * 256 + threadIdx.x;
  if (u >= total) return;
  f4_t v = sums[u];
  for (int i = 1; i < slices; ++i) v += sums[(int64_t)i * total + u];
  const uint32_t row = u / quads, col = 4 * (u - row * quads);
  store4_16<DT>(Y, (int64_t)row * ldy + col, N - col, v);
}

template <int FM, int WN, int DT>
void launch_tile(const Plan& p, const uint8_t* X, const uint8_t* ex, const uint8_t* W, const uint8_t* ew, int64_t M, int64_t N,
                 int64_t G, uint16_t* Y, int64_t ldy, float* ws, hipStream_t s) {
  const int64_t T = cdiv(M, 16 * FM) * cdiv(N, 64 * WN);
  float* const sums = p.slices > 1 ? ws : nullptr;
  {
    SlimKernelTimer timer("linear8_tile", s);
    SLIM_LAUNCH(timer, (k_linear8_tile<FM, WN, DT>), dim3((unsigned)(8 * cdiv(T, 8)), (unsigned)p.slices), dim3(256), s, X, ex, W, ew,
                M, N, (int)G, p.fours, Y, ldy, sums);
  }
  if (sums) {
    const int64_t quads = cdiv(N, 4), total = M * quads;
    SlimKernelTimer timer("linear8_sum", s);
    SLIM_LAUNCH(timer, k_linear8_sum<DT>, dim3((unsigned)cdiv(total, 256)), dim3(256), s, reinterpret_cast<const f4_t*>(sums), p.slices,
                (uint32_t)total, (uint32_t)quads, N, Y, ldy);
  }
}

// Blocks of up to 16 FM rows and NT weight tiles. Two tiles a block from 4096 columns on, where that leaves a block for
// every second CU: 5120 x 5120, M 1: 10.1 us against 10.9, M 16: 11.8 against 13.4; 2048 x 2048, M 1: 6.3 against 5.9.
template <int FM, int NT, int XT, int DT>
void launch_few_of(const void* X, const uint8_t* ex, int64_t ldx, const uint8_t* W, const uint8_t* ew, int64_t M, int64_t N,
                   int64_t K, uint16_t* Y, int64_t ldy, hipStream_t s) {
  SlimKernelTimer timer("linear8_few", s);
  SLIM_LAUNCH(timer, (k_linear8_few<FM, NT, 2, XT, DT>), dim3((unsigned)cdiv(N, 16 * NT)), dim3(512), s,
              reinterpret_cast<const uint8_t*>(X), ex, ldx, (int)K, W, ew, (int)M, N, (int)(q8_row(K) / 128), Y, ldy);
}
template <int XT, int DT>
void launch_few(const void* X, const uint8_t* ex, int64_t ldx, const uint8_t* W, const uint8_t* ew, int64_t M, int64_t N, int64_t K,
                uint16_t* Y, int64_t ldy, hipStream_t s) {
  if (N >= 4096) launch_few_of<1, 2, XT, DT>(X, ex, ldx, W, ew, M, N, K, Y, ldy, s);
  else launch_few_of<1, 1, XT, DT>(X, ex, ldx, W, ew, M, N, K, Y, ldy, s);
}

// X as codes.
template <int DT>
void launch(const Plan& p, const uint8_t* X, const uint8_t* ex, const uint8_t* W, const uint8_t* ew, int64_t M, int64_t N, int64_t K,
            uint16_t* Y, int64_t ldy, float* ws, hipStream_t s) {
  const int64_t G = q8_row(K) / 128;
  if (p.few == 1) return launch_few<SLIM_Q8_E4M3, DT>(X, ex, 0, W, ew, M, N, K, Y, ldy, s);
  if (p.few == 2) return launch_few_of<2, 2, SLIM_Q8_E4M3, DT>(X, ex, 0, W, ew, M, N, K, Y, ldy, s);
  if (p.few == 4) return launch_few_of<4, 1, SLIM_Q8_E4M3, DT>(X, ex, 0, W, ew, M, N, K, Y, ldy, s);
  switch (p.kind) {
    case 0: return launch_tile<16, 4, DT>(p, X, ex, W, ew, M, N, G, Y, ldy, ws, s);
    case 1: return launch_tile<12, 4, DT>(p, X, ex, W, ew, M, N, G, Y, ldy, ws, s);
    case 2: return launch_tile<8, 4, DT>(p, X, ex, W, ew, M, N, G, Y, ldy, ws, s);
    case 3: return launch_tile<8, 2, DT>(p, X, ex, W, ew, M, N, G, Y, ldy, ws, s);
    case 4: return launch_tile<4, 2, DT>(p, X, ex, W, ew, M, N, G, Y, ldy, ws, s);
    default: return launch_tile<4, 1, DT>(p, X, ex, W, ew, M, N, G, Y, ldy, ws, s);
  }
}

// Whether X is quantised in the product's launch (every block does it for itself): up to four rows whose codes fit in LDS.
bool quant_in_launch(int xdtype, int64_t M, int64_t K) { return xdtype != SLIM_Q8_E4M3 && M <= 4 && M * q8_row(K) <= kFewLds; }

}  // namespace

extern "C" int slim_linear8_workspace(int xdtype, int64_t M, int64_t N, int64_t K, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  const int rc = check_sizes(xdtype, M, N, K);
  if (rc != SLIM_OK) return rc;
  *bytes = 0;
  if (M == 0 || quant_in_launch(xdtype, M, K)) return SLIM_OK;
  const Plan p = plan(M, N, K);
  const TileKind& k = kTiles[p.kind];
  if (!p.few && !one_launch(8 * cdiv(cdiv(M, 16 * k.fm) * cdiv(N, 64 * k.wn), 8), 256)) return SLIM_EUNSUPPORTED;
  *bytes = p.bytes;
  if (xdtype != SLIM_Q8_E4M3) *bytes += code_bytes(M, K) + round256((size_t)M * (size_t)q8_exp_row(K));
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
  uint16_t* y = reinterpret_cast<uint16_t*>(Y);
  if (quant_in_launch(xdtype, M, K)) {
    const auto call = [&](auto xt, auto yt) {
      launch_few<decltype(xt)::value, decltype(yt)::value>(X, nullptr, ldx, codes, exps, M, N, K, y, ldy, s);
    };
    const auto to = [&](auto xt) {
      ydtype == SLIM_F16 ? call(xt, std::integral_constant<int, 0>{}) : call(xt, std::integral_constant<int, 1>{});
    };
    if (xdtype == SLIM_F16) to(std::integral_constant<int, SLIM_F16>{});
    else if (xdtype == SLIM_BF16) to(std::integral_constant<int, SLIM_BF16>{});
    else to(std::integral_constant<int, SLIM_F32>{});
    return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
  }
  const Plan p = plan(M, N, K);
  float* sums = reinterpret_cast<float*>(ws);
  if (!packed) {
    uint8_t* c = reinterpret_cast<uint8_t*>(ws);
    uint8_t* e = c + code_bytes(M, K);
    sums = reinterpret_cast<float*>(e + round256((size_t)M * (size_t)q8_exp_row(K)));
    const int q = slim_quant8(X, xdtype, M, K, ldx, c, e, stream);
    if (q != SLIM_OK) return q;
    xc = c;
    xe = e;
  }
  if (ydtype == SLIM_F16) launch<0>(p, xc, xe, codes, exps, M, N, K, y, ldy, sums, s);
  else launch<1>(p, xc, xe, codes, exps, M, N, K, y, ldy, sums, s);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
