// linear8_act.hip - 8-bit products that end in an activation, and its gradient by itself: slim_linear8_act, slim_bwd_dx8_act,
// slim_act_bwd.
//
// Forward: z = X W^T + bias, y = act(z) mul + residual. Backward: du = dh mul act'(u), dmul = dh act(u), dbias = sum over rows of
// du, with dh = dY W (the input gradient of the product that took y) or given. The products are linear8_product.h's; what they
// leave goes through ActRows (slim_act.h) in the same launch, so that neither z nor dh is written and read again: 8192 x 28672
// results in 16 bits would be 0.16 ms of memory traffic. Products whose reduction is in slices, and those whose blocks have no
// whole groups of 128 columns where those are needed (8-bit results, sums over rows), leave fp32 sums; k_act8_rows ends them.
#include <cstddef>

#include "linear8_product.h"
#include "slim_act.h"

namespace {

// fp32 sums [M][N up to 4].
struct SumRows {
  static constexpr bool kRows = false;
  static constexpr int kType = 0;
  float* sums;
  int64_t ld;
  SLIM_DEV void four(int64_t m, int64_t n, int64_t, f4_t v) const { *(SLIM_GLOBAL f4_t*)(sums + m * ld + n) = v; }
};

// Few rows. 1 x 11008 x 4096, silu and a gate's factor: 8 us (5.6 TB/s), as the bare product.
template <int FM, int NT, int XT, class Fin>
__global__ void __launch_bounds__(512)
k_act8_few(const uint8_t* __restrict__ X, const uint8_t* __restrict__ ex, int64_t ldx, int K, const uint8_t* __restrict__ W,
           const uint8_t* __restrict__ ew, int M, int64_t N, int G, Fin fin) {
  few_body<FM, NT, 2, XT>(X, ex, ldx, K, W, ew, M, N, G, fin);
}

// 4096 x 28672 x 8192 on one card: 673 to 712 us with nothing added (the bare product 645 to 712, by what ran before: power), with a bias
// relu 680, silu 688, gelu_tanh 695, gelu 729, gelu to 8 bits 742, its argument too 773; backward of silu from 8 bits 738, with a gate
// 794: bound in its end by the instructions of one wave a SIMD (tiles that start apart, so that their memory traffic does not meet,
// took as long).
// What ends the rows is some thirty scalars, which the loop has no registers for: they are read from the launch's arguments anew
// after it (a copy behind an opaque address, which the compiler cannot move up; held over the loop they were spilled).
template <class Fin>
struct TileCall {
  const uint8_t *X, *ex, *W, *ew;
  int64_t M, N;
  int G, fours;
  float* sums;
  Fin fin;
};
template <int FM, int WN, class Fin>
__global__ void __launch_bounds__(256, 1)
k_act8_tile(TileCall<Fin> c) {
#if defined(__HIP_DEVICE_COMPILE__)
  tile_body<FM, WN>(c.X, c.ex, c.W, c.ew, c.M, c.N, c.G, c.fours, c.sums, [] {
    typedef const __attribute__((address_space(4))) uint32_t* words_t;
    words_t at = (words_t)__builtin_amdgcn_kernarg_segment_ptr();       // the only argument starts it
    asm volatile("" : "+s"(at));
    static_assert(sizeof(Fin) % 4 == 0 && offsetof(TileCall<Fin>, fin) % 4 == 0);
    uint32_t w[sizeof(Fin) / 4];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Fin) / 4); ++i) w[i] = at[offsetof(TileCall<Fin>, fin) / 4 + i];
    Fin fin;
    __builtin_memcpy(&fin, w, sizeof(Fin));
    return fin;
  });
#endif
}

// Ends rows whose sums (`slices` of them, fp32 [M][N up to 4] each, added in slice order) or whose dh (16 bits) lie in memory: `lpr`
// lanes take a row of 8 lpr columns, a block the rows r0 .. r0 + per, two of a lane's in flight while two are ended.
// Bound by HBM: the gradient of gelu_tanh from 8 bits over 8192 x 28672, with sums over rows, 243 us (4.9 TB/s; four rows at a
// time without any ahead 268).
template <bool BWD, int DT, bool SUMS>
__global__ void __launch_bounds__(256, 2)
k_act8_rows(const void* __restrict__ src, int64_t ld, int slices, int64_t stride, int64_t M, int64_t N, int per, int lpr, uint32_t strips,
            ActRows<BWD, DT> fin) {
  __shared__ float red[4 * 512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t block = blockIdx.x / strips, strip = blockIdx.x - block * strips, r0 = block * per;
  const int64_t col = 8 * (strip * lpr + lane % lpr);
  const int rows = (int)(M - r0 < per ? M - r0 : per), step = 4 * (64 / lpr), at0 = wave * (64 / lpr) + lane / lpr;
  typename ActRows<BWD, DT>::Lane l;
  fin.begin(l, r0 + at0, step, col);
  const int todo = fin.todo();
  typedef typename ActRows<BWD, DT>::In In;
  constexpr int NB = 2;
  const auto turns = [&](auto whole) SLIM_INLINE {
    constexpr bool W = decltype(whole)::value;
    const auto there = [&](int row) { return W || (row < rows && l.n); };
    const auto load = [&](u32x4_t* d, In* in, int row) SLIM_INLINE {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        d[b] = u32x4_t{0, 0, 0, 0};
        if constexpr (!SUMS)
          if (there(row + step * b))
            d[b] = ActRows<BWD, DT>::load16(reinterpret_cast<const char*>(src) + 2 * ((r0 + row + step * b) * ld + col), W ? 8 : l.n);
      }
      fin.template load_rows<W, NB>(in, l, todo, step, rows - row);
    };
    u32x4_t d[NB];
    In in[NB];
    load(d, in, at0);
#pragma unroll 1
    for (int t = 0; t < rows; t += NB * step) {      // the same number of turns for every lane
      float f[NB][8];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if constexpr (SUMS) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[b][e] = 0.f;
          if (!there(t + at0 + step * b)) continue;
          const float* s = reinterpret_cast<const float*>(src) + (r0 + t + at0 + step * b) * ld + col;
          for (int i = 0; i < slices; ++i, s += stride) {
            const f4_t lo = *reinterpret_cast<const f4_t*>(s);
            const f4_t hi = W || l.n > 4 ? *reinterpret_cast<const f4_t*>(s + 4) : f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              f[b][e] += lo[e];
              f[b][4 + e] += hi[e];
            }
          }
        } else {
          act8_to_f(d[b], DT == 1, f[b]);
        }
      }
      u32x4_t dn[NB];
      In next[NB];
      if (t + NB * step < rows) load(dn, next, t + at0 + NB * step);
      __builtin_amdgcn_sched_barrier(0);
      fin.template end_rows<W, NB>(l, in, todo, step, rows - t - at0, f);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        d[b] = dn[b];
        in[b] = next[b];
      }
    }
  };
  // whole turns of whole columns need no bounds
  if (rows % (NB * step) == 0 && 8 * (strip + 1) * lpr <= N) turns(std::true_type{});
  else turns(std::false_type{});
  if (fin.sums_wanted()) {
    // over the row places of a wave, then over the waves in order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = l.s[e];
      if (lpr <= 32) v += __shfl_xor(v, 32, 64);
      if (lpr <= 16) v += __shfl_xor(v, 16, 64);
      if (lane < lpr) red[wave * 512 + 8 * lane + e] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * lpr; i += 256) {
      const int64_t c = 8 * strip * lpr + i;
      if (c < N) fin.put_sum(block, c, N, red[i] + red[512 + i] + red[1024 + i] + red[1536 + i]);
    }
  }
}

// Sums over the blocks of each column's parts, in an order of their own: 16 waves take every 16th, then wave by wave. OT: the type
// they leave in.
template <int OT>
__global__ void __launch_bounds__(1024)
k_act8_sums(const float* __restrict__ part, int64_t blocks, int64_t N, void* __restrict__ out) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + lane;
  float v = 0.f;
  if (col < N) {
#pragma unroll 4
    for (int64_t b = wave; b < blocks; b += 16) v += part[b * N + col];
  }
  red[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && col < N) {
    for (int i = 1; i < 16; ++i) v += red[i][lane];
    store_elem<OT>(out, col, v);
  }
}

// ------------------------------------------------------------------------------------- host
// How k_act8_rows covers M rows of N columns: lanes a row, strips side by side, rows a block. About 2048 blocks, of 16 rows a
// lane's turn at least.
struct RowPlan {
  int lpr, per;
  int64_t strips, blocks;
};
RowPlan row_plan(int64_t M, int64_t N) {
  RowPlan p;
  const int64_t eights = q8_row(N) / 8;
  p.lpr = eights <= 16 ? 16 : eights <= 32 ? 32 : 64;
  p.strips = cdiv(eights, p.lpr);
  const int64_t turn = 16 * (64 / p.lpr);
  p.per = (int)(cdiv(std::max<int64_t>(1, cdiv(M * p.strips, 2048)), turn) * turn);
  p.blocks = cdiv(M, p.per);
  return p;
}

template <bool BWD, int DT, bool SUMS>
void launch_rows(const void* src, int64_t ld, int slices, int64_t stride, int64_t M, const ActArgs& a, hipStream_t s) {
  const RowPlan p = row_plan(M, a.N);
  SlimKernelTimer timer("act8_rows", s);
  SLIM_LAUNCH(timer, (k_act8_rows<BWD, DT, SUMS>), dim3((unsigned)(p.strips * p.blocks)), dim3(256), s, src, ld, slices, stride, M, a.N, p.per,
              p.lpr, (uint32_t)p.strips, (ActRows<BWD, DT>{a}));
}

void launch_sums(const float* part, int64_t blocks, int64_t N, void* out, int dtype, hipStream_t s) {
  SlimKernelTimer timer("act8_sums", s);
  const dim3 grid((unsigned)cdiv(N, 64));
  if (dtype == SLIM_F32) SLIM_LAUNCH(timer, k_act8_sums<2>, grid, dim3(1024), s, part, blocks, N, out);
  else if (dtype == SLIM_BF16) SLIM_LAUNCH(timer, k_act8_sums<1>, grid, dim3(1024), s, part, blocks, N, out);
  else SLIM_LAUNCH(timer, k_act8_sums<0>, grid, dim3(1024), s, part, blocks, N, out);
}

}  // namespace

// The few kernel's blocks have 16 or 32 columns, the narrowest tile's 64.
SlimActPlan slim_act_plan(bool bwd, int xdtype, int64_t M, int64_t N, int64_t K, bool groups, bool sums) {
  const Plan p = plan(M, N, K, 3.5 + 2.0 * M * N * 4 / 4e6);      // the sums' way through memory, as tile_time's of one slice more
  const TileKind& k = kTiles[p.kind];
  SlimActPlan a{p.few, p.kind, p.slices, p.fours};
  a.direct = a.few ? !bwd && !groups : a.slices == 1 && k.wn > 1;
  a.sum_bytes = a.direct ? 0 : round256((size_t)a.slices * (size_t)M * (size_t)((N + 3) & ~int64_t(3)) * 4);
  a.blocks = a.direct ? cdiv(M, 16 * k.fm) : row_plan(M, N).blocks;
  a.part_bytes = sums ? round256((size_t)a.blocks * (size_t)N * 4) : 0;
  a.x_bytes = xdtype == SLIM_Q8_E4M3 ? 0 : code_bytes(M, K) + round256((size_t)M * (size_t)q8_exp_row(K));
  return a;
}

namespace {

struct Product {
  const uint8_t *X, *ex, *W, *ew;
  int64_t ldx, M, N, K;
};

template <int FM, int WN, class Fin>
void launch_act_tile(const SlimActPlan& p, const Product& d, float* sums, const Fin& fin, hipStream_t s) {
  const int64_t T = cdiv(d.M, 16 * FM) * cdiv(d.N, 64 * WN);
  SlimKernelTimer timer("act8_tile", s);
  SLIM_LAUNCH(timer, (k_act8_tile<FM, WN, Fin>), dim3((unsigned)(8 * cdiv(T, 8)), (unsigned)p.slices), dim3(256), s,
              (TileCall<Fin>{d.X, d.ex, d.W, d.ew, d.M, d.N, (int)(q8_row(d.K) / 128), p.fours, sums, fin}));
}
template <int FM, int NT, int XT, class Fin>
void launch_act_few(const Product& d, const Fin& fin, hipStream_t s) {
  SlimKernelTimer timer("act8_few", s);
  SLIM_LAUNCH(timer, (k_act8_few<FM, NT, XT, Fin>), dim3((unsigned)cdiv(d.N, 16 * NT)), dim3(512), s, d.X, d.ex, d.ldx, (int)d.K, d.W, d.ew,
              (int)d.M, d.N, (int)(q8_row(d.K) / 128), fin);
}
// XT as few_body's: other than codes only for few == 1.
template <int XT, class Fin>
void launch_few(int few, const Product& d, const Fin& fin, hipStream_t s) {
  if constexpr (XT == SLIM_Q8_E4M3) {
    if (few == 2) return launch_act_few<2, 2, XT>(d, fin, s);
    if (few == 4) return launch_act_few<4, 1, XT>(d, fin, s);
  }
  if (d.N >= 4096) launch_act_few<1, 2, XT>(d, fin, s);      // as slim_linear8's
  else launch_act_few<1, 1, XT>(d, fin, s);
}

template <bool BWD, int DT>
int launch_act(const SlimActPlan& a, const Product& d, float* sums, const ActArgs& args, hipStream_t s) {
  const ActRows<BWD, DT> fin{args};
  if (a.direct) {
    if constexpr (!BWD)
      if (a.few) {
        launch_few<SLIM_Q8_E4M3>(a.few, d, fin, s);
        return SLIM_OK;
      }
    switch (a.kind) {
      case 0: launch_act_tile<16, 4>(a, d, nullptr, fin, s); break;
      case 1: launch_act_tile<12, 4>(a, d, nullptr, fin, s); break;
      case 2: launch_act_tile<8, 4>(a, d, nullptr, fin, s); break;
      case 3: launch_act_tile<8, 2>(a, d, nullptr, fin, s); break;
      default: launch_act_tile<4, 2>(a, d, nullptr, fin, s); break;
    }
    return SLIM_OK;
  }
  const int64_t ld = (d.N + 3) & ~int64_t(3);
  const SumRows out{sums, ld};
  if (a.few) {
    launch_few<SLIM_Q8_E4M3>(a.few, d, out, s);
  } else {
    switch (a.kind) {
      case 3: launch_act_tile<8, 2>(a, d, sums, out, s); break;
      case 4: launch_act_tile<4, 2>(a, d, sums, out, s); break;
      case 5: launch_act_tile<4, 1>(a, d, sums, out, s); break;
      default: return SLIM_EUNSUPPORTED;      // wide tiles have no slices
    }
  }
  launch_rows<BWD, DT, true>(sums, ld, a.slices, d.M * ld, d.M, args, s);
  return SLIM_OK;
}

bool is_16(int t) { return t == SLIM_F16 || t == SLIM_BF16; }
bool is_float(int t) { return is_16(t) || t == SLIM_F32; }
size_t elem(int t) { return t == SLIM_F32 ? 4 : 2; }

// Operands and results in memory.
SlimRows rows_of(const void* p, int64_t M, int64_t N, int64_t ld, size_t bytes) { return {p, M, N * (int64_t)bytes, ld * (int64_t)bytes}; }
SlimRows codes_of(const void* p, int64_t M, int64_t N) { return {p, M, q8_row(N), q8_row(N)}; }
SlimRows exps_of(const void* p, int64_t M, int64_t N) { return {p, M, q8_exp_row(N), q8_exp_row(N)}; }
SlimRows vector_of(const void* p, int64_t N, size_t bytes) { return {p, 1, N * (int64_t)bytes, 0}; }

// Whether X's rows are turned into codes in the product's own launch (few rows of the results' type).
bool in_launch(bool bwd, int xdtype, int dtype, int64_t M, int64_t K, bool groups) {
  return !bwd && !groups && xdtype == dtype && M <= 4 && M * q8_row(K) <= kFewLds;
}

int product_workspace(bool bwd, int xdtype, int64_t M, int64_t N, int64_t K, int dtype, bool groups, bool sums, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  const int rc = check_sizes(xdtype, M, N, K);
  if (rc != SLIM_OK) return rc;
  if (!is_16(dtype)) return SLIM_EDTYPE;
  *bytes = 0;
  if (M == 0 || in_launch(bwd, xdtype, dtype, M, K, groups)) return SLIM_OK;
  const SlimActPlan a = slim_act_plan(bwd, xdtype, M, N, K, groups, sums);
  const TileKind& k = kTiles[a.kind];
  if (!a.few && !one_launch(8 * cdiv(cdiv(M, 16 * k.fm) * cdiv(N, 64 * k.wn), 8), 256)) return SLIM_EUNSUPPORTED;
  if (M > kMaxGroups8 / cdiv(N, 128)) return SLIM_EUNSUPPORTED;       // rows kept in 8 bits
  *bytes = a.x_bytes + a.sum_bytes + a.part_bytes;
  return SLIM_OK;
}

// What both entry points ask of the product's operands and of `need` bytes of workspace.
int check_product(const void* X, int xdtype, const uint8_t* xexps, const uint8_t* codes, const uint8_t* exps, size_t need, const void* ws,
                  size_t ws_bytes) {
  const bool packed = xdtype == SLIM_Q8_E4M3;
  if (!X || (packed && !xexps) || !codes || !exps) return SLIM_EINVAL;
  if (!slim_aligned_to(X, packed ? 16 : elem(xdtype)) || !slim_aligned16(xexps) || !slim_aligned16(codes) || !slim_aligned16(exps))
    return SLIM_EALIGN;
  if (need && (!ws || ws_bytes < need)) return SLIM_EWORKSPACE;
  if (need && !slim_aligned16(ws)) return SLIM_EALIGN;
  return SLIM_OK;
}

// The product of both entry points, of checked operands.
template <bool BWD>
int product(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t N, int64_t K, int64_t ldx, const uint8_t* codes,
            const uint8_t* exps, ActArgs args, int dtype, bool groups, void* dbias, void* ws, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  Product d{reinterpret_cast<const uint8_t*>(X), xexps, codes, exps, ldx, M, N, K};
  if (in_launch(BWD, xdtype, dtype, M, K, groups)) {
    if constexpr (!BWD) {
      if (dtype == SLIM_F16) launch_few<SLIM_F16>(1, d, ActRows<false, 0>{args}, s);
      else launch_few<SLIM_BF16>(1, d, ActRows<false, 1>{args}, s);
    }
    return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
  }
  const SlimActPlan a = slim_act_plan(BWD, xdtype, M, N, K, groups, dbias != nullptr);
  char* at = reinterpret_cast<char*>(ws);
  if (xdtype != SLIM_Q8_E4M3) {
    uint8_t* c = reinterpret_cast<uint8_t*>(at);
    uint8_t* e = c + code_bytes(M, K);
    const int q = slim_quant8(X, xdtype, M, K, ldx, c, e, stream);
    if (q != SLIM_OK) return q;
    d.X = c;
    d.ex = e;
  }
  float* const sums = reinterpret_cast<float*>(at + a.x_bytes);
  float* const part = reinterpret_cast<float*>(at + a.x_bytes + a.sum_bytes);
  args.part = dbias ? part : nullptr;
  const int rc = dtype == SLIM_F16 ? launch_act<BWD, 0>(a, d, sums, args, s) : launch_act<BWD, 1>(a, d, sums, args, s);
  if (rc != SLIM_OK) return rc;
  if (dbias) launch_sums(part, a.blocks, N, dbias, dtype, s);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

bool is_act(int act) { return act >= SLIM_ACT_NONE && act <= SLIM_ACT_SILU; }

// The backward's operands and results: N columns (dh's).
int check_bwd(int64_t N, int act, const void* U, int udtype, const uint8_t* uexps, int64_t ldu, const void* mul, const uint8_t* mulexps,
              int64_t ldmul, int dtype, const void* dU, int64_t lddu, const void* dmul, int64_t lddmul, bool none) {
  if (!is_16(dtype) || (udtype != dtype && udtype != SLIM_Q8_E4M3)) return SLIM_EDTYPE;
  const bool q8 = udtype == SLIM_Q8_E4M3;
  if (!is_act(act)) return SLIM_EINVAL;
  if (lddu < N || (dmul && lddmul < N) || (!q8 && ((U && ldu < N) || (mul && ldmul < N)))) return SLIM_ESHAPE;
  if (none) return SLIM_OK;
  if (!dU || (!U && (act != SLIM_ACT_NONE || dmul)) || (U && q8 && !uexps) || (mul && q8 && !mulexps) || (!mul != !dmul)) return SLIM_EINVAL;
  const size_t to = q8 ? 16 : 2;
  if ((U && !slim_aligned_to(U, to)) || (mul && !slim_aligned_to(mul, to)) || !slim_aligned_to(dU, 2) || (dmul && !slim_aligned_to(dmul, 2)))
    return SLIM_EALIGN;
  return SLIM_OK;
}

// Whether the backward's results may be written while U, mul and `src` (dH) are read: the lane that writes an element has read it in
// 16-bit operands before. 8-bit ones (and a product's operand `x` with exponents `xe`) have their elements elsewhere.
bool bwd_may_write(int64_t M, int64_t N, const ActArgs& a, const void* dbias, size_t bias_bytes, SlimRows src, SlimRows x, SlimRows xe) {
  const SlimRows du = rows_of(a.y, M, N, a.ldy, 2), dm = rows_of(a.w, M, N, a.ldw, 2), db = vector_of(dbias, N, bias_bytes);
  if (a.q8)
    return slim_may_write({du, dm, db}, {src}, {x, xe, codes_of(a.u, M, N), exps_of(a.u ? a.ue : nullptr, M, N), codes_of(a.mul, M, N),
                                                exps_of(a.mul ? a.me : nullptr, M, N)});
  return slim_may_write({du, dm, db}, {src, rows_of(a.u, M, N, a.ldu, 2), rows_of(a.mul, M, N, a.ldmul, 2)}, {x, xe});
}

ActArgs bwd_args(int64_t N, int act, const void* U, int udtype, const uint8_t* uexps, int64_t ldu, const void* mul, const uint8_t* mulexps,
                 int64_t ldmul, void* dU, int64_t lddu, void* dmul, int64_t lddmul) {
  ActArgs a{};
  a.act = act;
  a.q8 = udtype == SLIM_Q8_E4M3;
  a.N = N;
  a.u = U; a.ue = uexps; a.ldu = ldu;
  a.mul = mul; a.me = mulexps; a.ldmul = ldmul;
  a.y = dU; a.ldy = lddu;
  a.w = dmul; a.ldw = lddmul;
  return a;
}

}  // namespace

extern "C" int slim_linear8_act_workspace(int xdtype, int64_t M, int64_t N, int64_t K, int dtype, int q8, size_t* bytes) {
  return product_workspace(false, xdtype, M, N, K, dtype, q8 != 0, false, bytes);
}

extern "C" int slim_linear8_act(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t N, int64_t K, int64_t ldx,
                                const uint8_t* codes, const uint8_t* exps, int act, const void* bias, int bdtype, const void* mul,
                                int64_t ldmul, const void* residual, int64_t ldres, int dtype, int q8, void* Y, int64_t ldy,
                                uint8_t* yexps, void* pre, int64_t ldpre, uint8_t* preexps, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = slim_linear8_act_workspace(xdtype, M, N, K, dtype, q8, &need);
  if (rc != SLIM_OK) return rc;
  if (bias && !is_float(bdtype)) return SLIM_EDTYPE;
  if (!is_act(act)) return SLIM_EINVAL;
  if ((xdtype != SLIM_Q8_E4M3 && ldx < K) || (mul && ldmul < N) || (residual && ldres < N) || (!q8 && (ldy < N || (pre && ldpre < N))))
    return SLIM_ESHAPE;
  if (M == 0) return SLIM_OK;
  if (!Y || (q8 && (!yexps || (pre && !preexps)))) return SLIM_EINVAL;
  const size_t to = q8 ? 16 : 2;
  if (!slim_aligned_to(Y, to) || (pre && !slim_aligned_to(pre, to)) || (mul && !slim_aligned_to(mul, 2)) ||
      (residual && !slim_aligned_to(residual, 2)) || (bias && !slim_aligned_to(bias, elem(bdtype))))
    return SLIM_EALIGN;
  const int bad = check_product(X, xdtype, xexps, codes, exps, need, ws, ws_bytes);
  if (bad != SLIM_OK) return bad;
  // Blocks read X while others write. mul and residual are read element for element by the lane that writes Y and pre there, before
  // it does, so 16-bit results may take their very rows; 8-bit ones would lie over rows of other lanes.
  const bool packed = xdtype == SLIM_Q8_E4M3;
  const SlimRows x = packed ? codes_of(X, M, K) : rows_of(X, M, K, ldx, elem(xdtype)), xe = exps_of(packed ? xexps : nullptr, M, K);
  const SlimRows b = vector_of(bias, N, elem(bdtype)), m = rows_of(mul, M, N, ldmul, 2), r = rows_of(residual, M, N, ldres, 2);
  if (q8 ? !slim_may_write({codes_of(Y, M, N), exps_of(yexps, M, N), codes_of(pre, M, N), exps_of(pre ? preexps : nullptr, M, N)}, {}, {x, xe, b, m, r})
         : !slim_may_write({rows_of(Y, M, N, ldy, 2), rows_of(pre, M, N, ldpre, 2)}, {m, r}, {x, xe, b}))
    return SLIM_EINVAL;
  ActArgs a{};
  a.act = act;
  a.bdt = bdtype;
  a.q8 = q8 != 0;
  a.N = N;
  a.bias = bias;
  a.mul = mul; a.ldmul = ldmul;
  a.res = reinterpret_cast<const uint16_t*>(residual); a.ldres = ldres;
  a.y = Y; a.ye = yexps; a.ldy = ldy;
  a.w = pre; a.we = preexps; a.ldw = ldpre;
  return product<false>(X, xdtype, xexps, M, N, K, ldx, codes, exps, a, dtype, q8 != 0, nullptr, ws, stream);
}

extern "C" int slim_bwd_dx8_act_workspace(int dydtype, int64_t M, int64_t N, int64_t K, int dtype, int sums, size_t* bytes) {
  return product_workspace(true, dydtype, M, K, N, dtype, true, sums != 0, bytes);
}

extern "C" int slim_bwd_dx8_act(const void* dY, int dydtype, const uint8_t* dyexps, int64_t M, int64_t N, int64_t K, int64_t lddy,
                                const uint8_t* codesT, const uint8_t* expsT, int act, const void* U, int udtype, const uint8_t* uexps,
                                int64_t ldu, const void* mul, const uint8_t* mulexps, int64_t ldmul, int dtype, void* dU, int64_t lddu,
                                void* dmul, int64_t lddmul, void* dbias, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  int rc = slim_bwd_dx8_act_workspace(dydtype, M, N, K, dtype, dbias != nullptr, &need);
  if (rc != SLIM_OK) return rc;
  rc = check_bwd(K, act, U, udtype, uexps, ldu, mul, mulexps, ldmul, dtype, dU, lddu, dmul, lddmul, M == 0);
  if (rc != SLIM_OK) return rc;
  if (dydtype != SLIM_Q8_E4M3 && lddy < N) return SLIM_ESHAPE;
  if (dbias && !slim_aligned_to(dbias, 2)) return SLIM_EALIGN;
  if (M == 0) {
    if (dbias) launch_sums(nullptr, 0, K, dbias, dtype, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
  }
  rc = check_product(dY, dydtype, dyexps, codesT, expsT, need, ws, ws_bytes);
  if (rc != SLIM_OK) return rc;
  const ActArgs a = bwd_args(K, act, U, udtype, uexps, ldu, mul, mulexps, ldmul, dU, lddu, dmul, lddmul);
  // a dY of another type is read, turned into 8 bits in the workspace, before anything is written
  const bool packed = dydtype == SLIM_Q8_E4M3;
  if (!bwd_may_write(M, K, a, dbias, 2, SlimRows{}, codes_of(packed ? dY : nullptr, M, N), exps_of(packed ? dyexps : nullptr, M, N)))
    return SLIM_EINVAL;
  return product<true>(dY, dydtype, dyexps, M, K, N, lddy, codesT, expsT, a, dtype, true, dbias, ws, stream);
}

extern "C" int slim_act_bwd_workspace(int64_t M, int64_t K, int sums, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  if (M < 0 || K < 1 || K > kMaxRow8) return SLIM_ESHAPE;
  if (M > kMaxGroups8 / cdiv(K, 128)) return SLIM_EUNSUPPORTED;
  *bytes = 0;
  if (M == 0) return SLIM_OK;
  const RowPlan p = row_plan(M, K);
  if (!one_launch(p.strips * p.blocks, 256)) return SLIM_EUNSUPPORTED;
  if (sums && p.blocks > 1) *bytes = (size_t)p.blocks * (size_t)K * 4;      // one block's sums are dbias
  return SLIM_OK;
}

extern "C" int slim_act_bwd(const void* dH, int dtype, int64_t lddh, int64_t M, int64_t K, int act, const void* U, int udtype,
                            const uint8_t* uexps, int64_t ldu, const void* mul, const uint8_t* mulexps, int64_t ldmul, void* dU,
                            int64_t lddu, void* dmul, int64_t lddmul, float* dbias, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  int rc = slim_act_bwd_workspace(M, K, dbias != nullptr, &need);
  if (rc != SLIM_OK) return rc;
  rc = check_bwd(K, act, U, udtype, uexps, ldu, mul, mulexps, ldmul, dtype, dU, lddu, dmul, lddmul, M == 0);
  if (rc != SLIM_OK) return rc;
  if (lddh < K) return SLIM_ESHAPE;
  if (dbias && !slim_aligned_to(dbias, 4)) return SLIM_EALIGN;
  hipStream_t s = (hipStream_t)stream;
  if (M == 0) {
    if (dbias) launch_sums(nullptr, 0, K, dbias, SLIM_F32, s);
    return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
  }
  if (!dH) return SLIM_EINVAL;
  if (!slim_aligned_to(dH, 2)) return SLIM_EALIGN;
  if (need && (!ws || ws_bytes < need)) return SLIM_EWORKSPACE;
  if (need && !slim_aligned16(ws)) return SLIM_EALIGN;
  ActArgs a = bwd_args(K, act, U, udtype, uexps, ldu, mul, mulexps, ldmul, dU, lddu, dmul, lddmul);
  if (!bwd_may_write(M, K, a, dbias, 4, rows_of(dH, M, K, lddh, 2), SlimRows{}, SlimRows{})) return SLIM_EINVAL;
  const int64_t blocks = row_plan(M, K).blocks;
  a.part = !dbias ? nullptr : blocks > 1 ? reinterpret_cast<float*>(ws) : dbias;
  if (dtype == SLIM_F16) launch_rows<true, 0, false>(dH, lddh, 1, 0, M, a, s);
  else launch_rows<true, 1, false>(dH, lddh, 1, 0, M, a, s);
  if (dbias && blocks > 1) launch_sums(a.part, blocks, K, dbias, SLIM_F32, s);
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}
