// grad_w8.hip - the weight gradient from an 8-bit checkpoint of the activations: slim_grad_w8.
//
// D[k][n] = sum_m X[m][k] dY[m][n] (= grad W^T). The reduction runs along the stored rows of both operands, so a power of
// two for each row and group cannot be taken out of the sum: the codes are widened to dY's 16-bit type with their exponent
// on the way into LDS, and the products run on v_mfma_f32_32x32x16 with fp32 accumulators. X moves at half the bytes of a
// 16-bit activation.
//
// Widening is exact in bf16 (from 2^-130 on). fp16 holds 448 2^7 at most, so that where a block's rows have a larger exponent than 7 in a group
// of 128 columns, it lowers all of that group's exponents by `down`, as much as the largest needs, and multiplies the group's
// sums by 2^down at the end: finite gradients stay finite (fp16 activations come there from 63488 on, whose nearest code is
// 65536). Values below fp16's normal range are rounded to its steps, 2^-24, or 2^(down - 24) in such a group: less than 2^-39
// of the group's largest value.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <type_traits>

#include "slim_launch.h"
#include "slim_q8.h"
#include "slim_timing.h"

typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef short s4_t __attribute__((ext_vector_type(4)));

namespace {

constexpr int kWM = 32;       // rows of one chunk of the reduction
constexpr uint32_t kTop16 = 127 + 7;      // the largest exponent byte whose values fp16 holds

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

// Four consecutive positions k .. k + 3 of row n of the gradient: all of them, or the two that the pattern's byte for
// positions 8 (k / 8) .. keeps.
SLIM_DEV void store_grad4(float* gW, bool masked, uint32_t byte, int64_t n, int64_t k, int64_t K, f4_t v) {
  if (masked) {
    const uint32_t nib = (byte >> (k & 4)) & 0xFu, i0 = nib & 3u, i1 = nib >> 2;
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

// COUNT rows n, n + step, ... of a tile kept in LDS as [n][k] (SLOTS 16-byte slots a row, XOR-swizzled by the row), positions
// k .. k + 3 of each by this lane; `byte`: the pattern's byte for the positions 8 (k / 8) .. of each row.
template <int COUNT, int SLOTS>
SLIM_DEV void store_rows(float* gW, bool masked, const uint32_t (&byte)[COUNT], const f4_t* tile, int row, int step, int64_t n0, int64_t N,
                         int slot, int64_t k, int64_t K) {
  if (k >= K) return;
#pragma unroll
  for (int j = 0; j < COUNT; ++j) {
    const int i = row + j * step;
    if (n0 + i < N) store_grad4(gW, masked, byte[j], n0 + i, k, K, tile[i * SLOTS + (slot ^ (i & (SLOTS - 1)))]);
  }
}

// ------------------------------------------------------------------------------------- small layers
// TK (k) x 128 (n) tiles over a slice of the rows, eight waves in groups of TK / 32 that each hold the whole tile, 64 x 64 a
// wave: of each chunk of 64 rows a group takes its share (32 or 16), and the groups' sums are added through LDS at the end, in
// a fixed order. Both operands go through registers, where X is widened (and dY's rows may start anywhere), into two LDS slots;
// registers are loaded two chunks ahead of the slots. One barrier a chunk. A split launch writes its sums as one array a
// slice, which k_wgrad8_sum adds in slice order.
// TK 128: two blocks a CU hide each other's LDS and barriers. TK 64: for layers of so few tiles that a block stands alone
// on its CU anyway, where reads, products and writes of a chunk follow one another: half of each, on twice the CUs. 999 x 2051 x
// 768 14.7 us in bf16 and 15.2 in fp16 for a launch by itself, 13.3 and 13.8 where calls follow each other, 0.5 us a chunk of 64
// rows; 64 x 28672 x 8192 226 us with TK 128, of which writing the result is 184. TK 64 has one block a CU and no read of LDS in
// flight under its products: of the registers that a block alone on its CU could have, it uses half.
template <int DT, int HI>
SLIM_DEV uint32_t widen2(uint32_t c, float s);

// Barrier of a block's LDS accesses that leaves loads from memory in flight.
SLIM_DEV void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// fp16: what the exponents of a group, or of GROUPS = 2 next to each other, are lowered by, found by a block of THREADS threads
// from their bytes (the first at xe + at, a multiple of GROUPS, for `rows` rows ge bytes apart, ge a multiple of four). FLY loads a
// thread are issued at construction and, for most calls all there are, land while the block's first operands are on their way.
template <int THREADS, int FLY, int GROUPS>
struct Lowered {
  uint32_t b[FLY], top[GROUPS] = {};
  SLIM_DEV void load(const uint8_t* xe, uint32_t at, uint32_t ge, int64_t rows) {
    const rsrc_t r = make_rsrc(xe, rows * ge);          // rows past the last read as zero
    const uint32_t o = threadIdx.x * ge + at;
#pragma unroll
    for (int i = 0; i < FLY; ++i) {
      if constexpr (GROUPS == 2) b[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, o + i * THREADS * ge, 0, 0);
      else b[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, o + i * THREADS * ge, 0, 0);
    }
  }
  SLIM_DEV void take() {
#pragma unroll
    for (int i = 0; i < FLY; ++i)
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) top[g] = max(top[g], b[i] >> (8 * g) & 255u);
  }
  SLIM_DEV Lowered(const uint8_t* xe, uint32_t at, uint32_t ge, int64_t rows) {
    load(xe, at, ge, rows);
    while (rows > FLY * THREADS) {
      take();
      rows -= FLY * THREADS;
      xe += (int64_t)(FLY * THREADS) * ge;
      load(xe, at, ge, rows);
    }
  }
  // `part`: LDS of GROUPS THREADS / 64 words that nothing else reads or writes up to the block's next barrier
  SLIM_DEV void get(uint32_t* part, uint32_t (&down)[GROUPS]) {
    take();
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      top[g] = wave_max_u32(top[g]);
      if ((threadIdx.x & 63) == 0) part[g * (THREADS / 64) + (threadIdx.x >> 6)] = top[g];
    }
    sync_lds();
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) top[g] = max(top[g], part[g * (THREADS / 64) + w]);
      down[g] = (uint32_t)__builtin_amdgcn_readfirstlane((int)__builtin_elementwise_sub_sat(top[g], kTop16));
    }
  }
};

template <int DT, int TK>
__global__ void __launch_bounds__(512, 4)
k_wgrad8(const uint16_t* __restrict__ dY, int64_t lddy, int64_t cols, const uint8_t* __restrict__ xc, const uint8_t* __restrict__ xe,
         int64_t M, int64_t N, int64_t K, const uint8_t* __restrict__ meta, float* __restrict__ gW, int64_t slice, int64_t slice_out) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kRows = 2 * kWM, kAhead = 2, kGroups = 256 / TK, kSteps = 4 / kGroups, kSlots = TK / 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[4 * kRows * 256];      // X slots, dY slots; at the end the sums
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t Kp = q8_row(K), Ge = q8_exp_row(K);
  const uint32_t tk = (uint32_t)((K + TK - 1) / TK), nt = blockIdx.x / tk;
  const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane((int)nt) * 128;
  const int64_t k0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x - nt * tk)) * TK;
  const int64_t mb = blockIdx.y * slice, me = mb + slice < M ? mb + slice : M;
  gW += blockIdx.y * slice_out;
  // staging: row tid / 8 of the chunk, columns 16 (tid % 8) .. + 15 of dY, TK / 8 (tid % 8) .. of X
  const int row = tid >> 3, col = 16 * (tid & 7), xcol = TK / 8 * (tid & 7);
  const int nleft = (int)(cols - n0 - col < 16 ? cols - n0 - col : 16);     // cols: readable columns of dY, at least 16
  struct Stage {
    u32x4_t y0, y1;
    std::conditional_t<TK == 128, u32x4_t, u32x2_t> c;
    uint32_t e;
  };
  // the next chunk's row of this thread: rows are loaded in order
  int left = (int)(me - mb) - row, to_last = (int)(M - 1 - mb) - row;
  int64_t at = (mb + row) * lddy + n0 + col;
  // X by resources that move on with the chunk and end with the slice: rows past it read as zero
  const uint32_t xo = (uint32_t)row * (uint32_t)Kp + (uint32_t)(k0 + xcol), eo = (uint32_t)row * (uint32_t)Ge + (uint32_t)(k0 / 128);
  int64_t xm = mb;
  auto load = [&](Stage& S) {
    S.y0 = S.y1 = u32x4_t{0, 0, 0, 0};
    const rsrc_t rx = make_rsrc(xc + xm * Kp, (me - xm) * Kp);
    if constexpr (TK == 128) S.c = __builtin_amdgcn_raw_buffer_load_b128(rx, xo, 0, 0);
    else S.c = __builtin_amdgcn_raw_buffer_load_b64(rx, xo, 0, 0);
    S.e = __builtin_amdgcn_raw_buffer_load_b8(make_rsrc(xe + xm * Ge, (me - xm) * Ge), eo, 0, 0);
    xm += kRows;
    if (left > 0 && nleft > 0) {
      // past N the next row's values do no harm (results there are not stored); the last row's last piece is taken 16 values
      // from its end (N >= 16) and moved into place
      const int past = to_last == 0 ? 16 - nleft : 0;
      const uint16_t* p = dY + (at - past);
      __builtin_memcpy(&S.y0, p, 16);
      __builtin_memcpy(&S.y1, p + 8, 16);
      if (past) {
        if (past & 8) S.y0 = S.y1;
        if (past & 4) S.y0 = u32x4_t{S.y0[2], S.y0[3], S.y1[0], S.y1[1]}, S.y1 = u32x4_t{S.y1[2], S.y1[3], 0, 0};
        if (past & 2) S.y0 = u32x4_t{S.y0[1], S.y0[2], S.y0[3], S.y1[0]}, S.y1 = u32x4_t{S.y1[1], S.y1[2], S.y1[3], 0};
        if (past & 1) {
          S.y0 = u32x4_t{S.y0[0] >> 16 | S.y0[1] << 16, S.y0[1] >> 16 | S.y0[2] << 16, S.y0[2] >> 16 | S.y0[3] << 16,
                         S.y0[3] >> 16 | S.y1[0] << 16};
          S.y1 = u32x4_t{S.y1[0] >> 16 | S.y1[1] << 16, S.y1[1] >> 16 | S.y1[2] << 16, S.y1[2] >> 16 | S.y1[3] << 16, S.y1[3] >> 16};
        }
      }
    }
    left -= kRows;
    to_last -= kRows;
    at += kRows * lddy;
    asm volatile("" : "+v"(at));       // one offset, not one for each chunk of a round (and no pointer, whose loads would be generic)
  };
  uint8_t* const lx = lds + lds_at(row, xcol);
  uint8_t* const ly = lds + 2 * (kRows * 256) + lds_at(row, col);
  uint32_t down[1] = {0};
  auto put = [&](const Stage& S, int z) {
    uint8_t* x = lx + z * (kRows * 256);
    uint8_t* y = ly + z * (kRows * 256);
    *reinterpret_cast<u32x4_t*>(y) = S.y0;
    *reinterpret_cast<u32x4_t*>(y + 16) = S.y1;
    const float s = q8_pow2(DT == 0 ? __builtin_elementwise_sub_sat(S.e, down[0]) : S.e);
#pragma unroll
    for (int h = 0; h < TK / 64; ++h)
      *reinterpret_cast<u32x4_t*>(x + 16 * h) = u32x4_t{widen2<DT, 0>(S.c[2 * h], s), widen2<DT, 1>(S.c[2 * h], s),
                                                        widen2<DT, 0>(S.c[2 * h + 1], s), widen2<DT, 1>(S.c[2 * h + 1], s)};
  };
  f16_t acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i >> 1][i & 1][e] = 0.f;
  const int G = lane >> 4, q = lane & 15, grp = wave / (TK / 32);
  const int wk = TK == 128 ? 64 * (wave & 1) : 0, wn = 64 * ((TK == 128 ? wave >> 1 : wave) & 1);
  const int rr = 16 * kSteps * grp + 8 * (G >> 1) + (q >> 2), cr = 16 * (G & 1) + 4 * (q & 3);
  const uint8_t* ax[2] = {lds + lds_at(rr, wk + cr), lds + lds_at(rr, wk + 32 + cr)};
  const uint8_t* by[2] = {lds + 2 * (kRows * 256) + lds_at(rr, wn + cr), lds + 2 * (kRows * 256) + lds_at(rr, wn + 32 + cr)};
  Stage S[kAhead];
  // a chunk in slot j % 2; after its barrier no wave reads the other slot, which the next chunk takes
  auto chunk = [&](auto jc) {
    constexpr int j = decltype(jc)::value, z = j & 1;
    sync_lds();
    put(S[(j + 1) % kAhead], z ^ 1);
    load(S[(j + 1) % kAhead]);
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      __builtin_amdgcn_sched_barrier(0);        // one step's operands at a time: 128 registers for two blocks a CU
      u32x2_t a[2][2], b[2][2];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          a[f][i] = read_tr(ax[f] + z * (kRows * 256) + st * 4096 + i * 1024);      // 16 st + 4 i rows on: the same swizzle
          b[f][i] = read_tr(by[f] + z * (kRows * 256) + st * 4096 + i * 1024);
        }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) acc[x][y] = mfma_acc<DT>(a[x][0], a[x][1], b[y][0], b[y][1], acc[x][y]);
    }
  };
  if constexpr (DT == 0) {
    Lowered<512, 4, 1> l(xe + mb * Ge, (uint32_t)(k0 / 128), (uint32_t)Ge, me - mb);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(S[i]);
    __builtin_amdgcn_sched_barrier(0);
    l.get(reinterpret_cast<uint32_t*>(lds + kRows * 256), down);     // the second slot, written after the next barrier
  } else {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(S[i]);
  }
  put(S[0], 0);
  load(S[0]);
  // chunks past the last are zeros
  for (int64_t m = mb; m < me; m += kAhead * kRows) {
    chunk(std::integral_constant<int, 0>{});
    chunk(std::integral_constant<int, 1>{});
  }
  // what this thread stores, and the pattern's bytes for it, on their way while the sums are added
  const int slot = tid & (kSlots - 1), r0 = tid / kSlots;
  const int64_t k = k0 + 4 * slot;
  uint32_t byte[TK / 16];
  if (meta)
#pragma unroll
    for (int j = 0; j < TK / 16; ++j) {
      const int64_t n = n0 + r0 + j * (512 / kSlots);
      byte[j] = meta[(n < N ? n : N - 1) * (K / 8) + (k < K ? k : K - 1) / 8];
    }
  // The tile as [n][k] in LDS (16-byte slots XOR-swizzled by n): the groups' sums, last group first, which leave in whole
  // rows.
  __syncthreads();
  f4_t* const tile = reinterpret_cast<f4_t*>(lds);
  const int nl = wn + (lane & 31), sl = wk / 4 + (lane >> 5);
#pragma unroll
  for (int g = kGroups - 1; g >= 0; --g) {
    if (grp == g) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const f16_t& c = acc[i >> 3][(i >> 2) & 1];
        f4_t& t = tile[(nl + 32 * ((i >> 2) & 1)) * kSlots + ((sl + 8 * (i >> 3) + 2 * (i & 3)) ^ (nl & (kSlots - 1)))];
        f4_t v = {c[4 * (i & 3)], c[4 * (i & 3) + 1], c[4 * (i & 3) + 2], c[4 * (i & 3) + 3]};
        if constexpr (DT == 0) v *= q8_pow2(127 + down[0]);
        if (g == kGroups - 1) t = v;
        else t += v;
      }
    }
    __syncthreads();
  }
  store_rows<TK / 16, kSlots>(gW, meta != nullptr, byte, tile, r0, 512 / kSlots, n0, N, slot, k, K);
#endif
}

// The slices' sums, in slice order; four values a thread.
__global__ void __launch_bounds__(256)
k_wgrad8_sum(const float* __restrict__ part, int64_t slices, int64_t slice_out, int64_t count, float* __restrict__ gW) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= count) return;
  f4_t v = *reinterpret_cast<const f4_t*>(part + i);       // arrays of whole 16 bytes
  for (int64_t s = 1; s < slices; ++s) v += *reinterpret_cast<const f4_t*>(part + s * slice_out + i);
  if (i + 4 <= count) {
    *reinterpret_cast<f4_t*>(gW + i) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (i + e < count) gW[i + e] = v[e];
  }
}

// Rows of dY moved to 16-byte aligned ones (16 columns a thread), for the direct loads of the wide kernel.
__global__ void __launch_bounds__(256)
k_align_rows(const uint16_t* __restrict__ dY, int64_t lddy, uint32_t N, uint32_t pieces, uint32_t total, uint16_t* __restrict__ out) {
  const uint32_t u = blockIdx.x * 256 + threadIdx.x;
  if (u >= total) return;
  const uint32_t row = u / pieces, col = (u - row * pieces) * 16;
  const uint16_t* p = dY + (int64_t)row * lddy + col;
  uint16_t* o = out + ((int64_t)row * pieces * 16 + col);
  if (col + 16 <= N) {
    u32x4_t a, b;
    __builtin_memcpy(&a, p, 16);
    __builtin_memcpy(&b, p + 8, 16);
    *reinterpret_cast<u32x4_t*>(o) = a;
    *reinterpret_cast<u32x4_t*>(o + 8) = b;
  } else {
    for (uint32_t e = 0; e < 16; ++e) o[e] = col + e < N ? p[e] : (uint16_t)0;
  }
}

// ------------------------------------------------------------------------------------- large layers
// c += a b, written out so that the sum stays in its accumulation registers (the compiler moves 256 of them around a loop
// that has no others free). The operands were waited for; the sum was last written 15 products ago.
template <int DT>
SLIM_DEV void mfma_in_place(f16_t& c, u32x4_t a, u32x4_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (DT == 1) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
#endif
}

// Two of four codes times s as a pair of 16-bit values; s is a power of two, of which the instruction takes the exponent.
template <int DT, int HI>
SLIM_DEV uint32_t widen2(uint32_t c, float s) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (DT == 1) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, HI));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, s, HI));
#else
  return 0;
#endif
}

template <int N, int I = 0, class F>
SLIM_DEV void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, I + 1>(f);
  }
}

// byte offset of 16-bit column c of row r in 512-byte LDS rows, swizzled as lds_at
SLIM_DEV uint32_t lds_at_wide(int r, int c) {
  return (uint32_t)r * 512u + ((uint32_t)((c >> 4) ^ (2 * (r & 3))) << 5) + (uint32_t)((c & 15) * 2);
}

// 256 (k) x 256 (n) tiles, four waves of 128 x 128 (4 x 4 fragments, all accumulation registers of a SIMD's one wave): per
// 16 rows of the reduction a CU reads 32 KiB of operands from LDS for 512 cycles of products, half of what LDS delivers.
// A ring of four slots of 32 rows (16 KiB of dY, 16 KiB of widened X). dY, whose rows are 16-byte aligned, goes to LDS by
// direct loads three chunks ahead; X's codes are loaded four chunks ahead, widened and written to LDS two chunks ahead. One
// barrier a chunk, between its two 16-row steps, whose operands are read while the step before is multiplied. Columns past N
// and K read what lies there or zero; their results are not stored.
// Bound by the matrix unit, busy for 65 % of the cycles at the 1.6 GHz that the card then keeps (LDS for 33 %), and by its waits
// for operands: 8192 x 8192 x 8192 in bf16 865 to 900 us by card (1.22 to 1.27 PFLOP/s; a library product of bf16 operands 1.23), in
// fp16 2 % more; 8192 x 28672 x 8192 at kept positions 2.9 to 3.2 ms (1.2 to 1.3). Over few rows the first loads and last stores of
// every round of tiles show: 512 x 28672 x 8192 343 us (fp16 356), of which writing the result is 184; at kept positions 311.
template <int DT>
__global__ void __launch_bounds__(256, 1)
k_wgrad8_wide(const uint16_t* __restrict__ dY, int64_t lddy, const uint8_t* __restrict__ xc, const uint8_t* __restrict__ xe,
              int64_t M, int64_t N, int64_t K, const uint8_t* __restrict__ meta, float* __restrict__ gW) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr uint32_t kSlot = kWM * 512, kY = 4 * kSlot;
  __shared__ __attribute__((aligned(16))) uint8_t lds[8 * kSlot];
  __shared__ __attribute__((aligned(16))) uint8_t pattern[256][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = 128 * (wave & 1), wn = 128 * (wave >> 1);
  const uint32_t Kp = (uint32_t)q8_row(K), Ge = (uint32_t)q8_exp_row(K);
  // XCD-aware order (block b on XCD b % 8): bands of four n tiles, k tile by k tile
  const uint32_t tn = (uint32_t)((N + 255) / 256), tk = (uint32_t)((K + 255) / 256), T = tn * tk, Q = (T + 7) / 8;
  const uint32_t pos = (blockIdx.x % 8) * Q + blockIdx.x / 8;
  if (pos >= T) return;
  const uint32_t band = pos / (4 * tk), q0 = pos - band * 4 * tk, width = tn - band * 4 < 4 ? tn - band * 4 : 4, kt = q0 / width;
  const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(band * 4 + q0 - kt * width)) * 256;
  const int64_t k0 = (int64_t)__builtin_amdgcn_readfirstlane((int)kt) * 256;
  const int nch = (int)((M + kWM - 1) / kWM);

  // the pattern's bytes of one row of the tile a thread (past a row's end the next row's, which no result asks for)
  u32x4_t pat[2] = {};
  if (meta) {
    const int64_t bytes = N * (K / 8), at = (n0 + tid < N ? n0 + tid : N - 1) * (K / 8) + k0 / 8;
    if (at + 32 <= bytes) {
      __builtin_memcpy(pat, meta + at, 32);
    } else {
#pragma unroll
      for (int b = 0; b < 32; ++b) pat[b >> 4][(b >> 2) & 3] |= (uint32_t)(at + b < bytes ? meta[at + b] : 0) << (8 * (b & 3));
    }
  }

  // direct loads of dY: four pieces of 1 KiB (two rows) a wave; lane L writes LDS bytes 16 L of its piece, row L / 32,
  // physical slot L % 32, which holds logical slot (L % 32) ^ 4 (row % 4)
  uint32_t yo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 8 * wave + 2 * i + (lane >> 5), ls = (lane & 31) ^ (4 * (row & 3));
    yo[i] = ((uint32_t)row * (uint32_t)lddy + (uint32_t)(n0 + 8 * ls)) * 2u;
  }
  // Loads of chunk c: resources start at the group of four chunks being worked on, so that 32-bit offsets do for operands of
  // any size, and end with the operand, so that rows past M read as zero. A chunk past the last gets an offset past every
  // resource (the last group's are below 2 GiB) and reads as zero too, without a memory access; its uniform offset is 0,
  // since the bounds check takes the uniform offset off the resource's size. M >= 1.
  const uint32_t ystep = (uint32_t)(kWM * 2) * (uint32_t)lddy, xstep = kWM * Kp, estep = kWM * Ge;
  rsrc_t ry, rx, re;
  int c0 = 0;
  auto rebase = [&](int c) {
    const int64_t m = (int64_t)c * kWM, left = M - m;
    c0 = c;
    // whole 32-bit words, by which the bounds are checked: an odd N ends inside one (lddy is even)
    ry = make_rsrc(dY + m * lddy, ((left - 1) * lddy + N + (N & 1)) * 2);
    rx = make_rsrc(xc + m * Kp, left * Kp);
    re = make_rsrc(xe + m * Ge, left * Ge);
  };
  auto in_group = [&](int c) { return c < nch ? (uint32_t)(c - c0) : 0u; };
  auto or_past = [&](int c, uint32_t o) { return c < nch ? o : 0x80000000u; };
  auto issue_y = [&](int c, auto zc, auto ic) {
    constexpr int i = decltype(ic)::value;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(ry, (lds_ptr_t)&lds[kY + decltype(zc)::value * kSlot + (uint32_t)(4 * wave + i) * 1024u], 16,
                                             or_past(c, yo[i]), in_group(c) * ystep, 0, 0);
  };
  // X through registers: rows tid / 16 and 16 more, 16 columns from 16 (tid % 16) on
  const int sr = tid >> 4, scol = 16 * (tid & 15);
  const uint32_t kc = (uint32_t)(k0 + scol < Kp ? k0 + scol : Kp - 16);
  uint32_t xo[2], eo[2], xw[2][2];
  const uint32_t lb = (uint32_t)(uintptr_t)(lds_ptr_t)&lds[0];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    xo[j] = (uint32_t)(sr + 16 * j) * Kp + kc;
    eo[j] = (uint32_t)(sr + 16 * j) * Ge + kc / 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) xw[j][h] = lb + lds_at_wide(sr + 16 * j, scol) + 16u * h;
  }
  struct Stage {
    u32x4_t x[2];
    uint32_t e[2];
  };
  auto load_x = [&](Stage& S, int c, auto jc) {
    constexpr int j = decltype(jc)::value;
    const uint32_t g = in_group(c);
    S.x[j] = __builtin_amdgcn_raw_buffer_load_b128(rx, or_past(c, xo[j]), g * xstep, 0);
    S.e[j] = __builtin_amdgcn_raw_buffer_load_b8(re, or_past(c, eo[j]), g * estep, 0);
  };
  // step i (0 .. 15) of a chunk's widening: two codes, and after each eighth the 16 bytes to LDS
  uint32_t down[2] = {0, 0}, low = 0;       // of the tile's two groups, and of this thread's columns
  u32x4_t wide;
  auto put_x = [&](const Stage& S, auto zc, auto ic) {
    constexpr uint32_t off = decltype(zc)::value * kSlot;
    constexpr int i = decltype(ic)::value, j = i >> 3, h = (i >> 2) & 1, e = i & 3;
    wide[e] = widen2<DT, e & 1>(S.x[j][2 * h + (e >> 1)], q8_pow2(DT == 0 ? __builtin_elementwise_sub_sat(S.e[j], low) : S.e[j]));
    if constexpr (e == 3) {
      const uint32_t at = xw[j][h];
      const u32x4_t v = wide;
      asm volatile("ds_write_b128 %0, %1 offset:%2" :: "v"(at), "v"(v), "i"(off) : "memory");
    }
  };

  f16_t acc[4][4];
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.f;
  // per-lane addresses of the transposed reads in slot 0, step 0 (lane mapping as in k_wgrad8)
  const int Gl = lane >> 4, ql = lane & 15, rr = 8 * (Gl >> 1) + (ql >> 2), cr = 16 * (Gl & 1) + 4 * (ql & 3);
  uint32_t ax[4][2], by[4][2];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      ax[f][j] = lb + lds_at_wide(rr + 4 * j, wk + 32 * f + cr);
      by[f][j] = lb + kY + lds_at_wide(rr + 4 * j, wn + 32 * f + cr);
    }
  struct Frags {
    u32x2_t a[4][2], b[4][2];
  };
  auto rd = [](u32x2_t& v, uint32_t at, auto oc) {
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(at), "i"(decltype(oc)::value));
  };
  // read i (0 .. 15) of a step: fragments of dY and X in the order the products need them
  auto read_i = [&](Frags& F, auto ic, auto oc) {
    constexpr int i = decltype(ic)::value, f = i >> 2, j = i & 1;
    if constexpr (i & 2) rd(F.a[f][j], ax[f][j], oc);
    else rd(F.b[f][j], by[f][j], oc);
  };
  auto landed = [](Frags& F) {
    asm volatile("s_waitcnt lgkmcnt(0)"
                 : "+v"(F.a[0][0]), "+v"(F.a[0][1]), "+v"(F.a[1][0]), "+v"(F.a[1][1]), "+v"(F.a[2][0]), "+v"(F.a[2][1]),
                   "+v"(F.a[3][0]), "+v"(F.a[3][1]), "+v"(F.b[0][0]), "+v"(F.b[0][1]), "+v"(F.b[1][0]), "+v"(F.b[1][1]),
                   "+v"(F.b[2][0]), "+v"(F.b[2][1]), "+v"(F.b[3][0]), "+v"(F.b[3][1]));
  };
  // The 16 products of the step in F; before each of the first eight two reads of the next step (at offset oc) into Nx, and
  // before product i the work of extra(i): a product takes 32 cycles, in which a wave issues about seven more instructions,
  // so the loads, widenings and writes of the chunks to come are spread over the products.
  auto step = [&](const Frags& F, Frags& Nx, auto oc, auto&& extra) {
    each<16>([&](auto ic) {
      constexpr int i = decltype(ic)::value, x = i >> 2, y = i & 3;
      if constexpr (i < 8) {
        read_i(Nx, std::integral_constant<int, 2 * i>{}, oc);
        read_i(Nx, std::integral_constant<int, 2 * i + 1>{}, oc);
      }
      extra(ic);
      __builtin_amdgcn_sched_barrier(0);
      const u32x4_t av = {F.a[x][0][0], F.a[x][0][1], F.a[x][1][0], F.a[x][1][1]};
      const u32x4_t bv = {F.b[y][0][0], F.b[y][0][1], F.b[y][1][0], F.b[y][1][1]};
      mfma_in_place<DT>(acc[x][y], av, bv);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  Frags A, B;
  Stage S[2];
  // Chunk c in slot z = c % 4. At its barrier dY of chunk c + 1 has landed for this wave once only the loads issued after it
  // are outstanding (X of chunk c + 2, dY of c + 2, X of c + 3: 12), and this wave's part of X, written a chunk ago, is in
  // LDS; after it no wave reads chunk c - 1, whose slot chunk c + 3 takes.
  auto chunk = [&](int c, auto zc) {
    constexpr int z = decltype(zc)::value;
    step(A, B, std::integral_constant<uint32_t, z * kSlot + 16 * 512>{}, [&](auto ic) {
      constexpr int i = decltype(ic)::value;
      put_x(S[z & 1], std::integral_constant<int, (z + 2) % 4>{}, ic);
    });
    landed(B);
    __builtin_amdgcn_s_waitcnt(vmcnt_wait(12));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    step(B, A, std::integral_constant<uint32_t, ((z + 1) % 4) * kSlot>{}, [&](auto ic) {
      constexpr int i = decltype(ic)::value;
      if constexpr (i >= 8 && i < 12) issue_y(c + 3, std::integral_constant<int, (z + 3) % 4>{}, std::integral_constant<int, i - 8>{});
      if constexpr (i == 13) load_x(S[z & 1], c + 4, I0{});
      if constexpr (i == 15) load_x(S[z & 1], c + 4, I1{});
    });
    landed(A);
  };
  rebase(0);
  auto first = [&] {
    each<4>([&](auto ic) { issue_y(0, I0{}, ic); });
    each<4>([&](auto ic) { issue_y(1, I1{}, ic); });
    each<4>([&](auto ic) { issue_y(2, I2{}, ic); });
    each<2>([&](auto jc) { load_x(S[0], 0, jc); });
    each<2>([&](auto jc) { load_x(S[1], 1, jc); });
  };
  if constexpr (DT == 0) {
    Lowered<256, 8, 2> l(xe, (uint32_t)(k0 / 128), Ge, M);
    __builtin_amdgcn_sched_barrier(0);
    first();
    __builtin_amdgcn_sched_barrier(0);
    l.get(reinterpret_cast<uint32_t*>(&pattern[0][0]), down);        // (written after the last product)
    low = down[(tid >> 3) & 1];
  } else {
    first();
  }
  each<16>([&](auto ic) { put_x(S[0], I0{}, ic); });
  each<16>([&](auto ic) { put_x(S[1], I1{}, ic); });
  each<2>([&](auto jc) { load_x(S[0], 2, jc); });
  each<2>([&](auto jc) { load_x(S[1], 3, jc); });
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_waitcnt(vmcnt_wait(0));
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  each<16>([&](auto ic) { read_i(A, ic, std::integral_constant<uint32_t, 0>{}); });
  landed(A);
  asm volatile("" : "+v"(pat[0]), "+v"(pat[1]));          // loaded by now
  int c = 0;
  do {                  // at least once: no way around the loop, on which the sums would be moved
    if (c) rebase(c);
    // chunks past the last are zeros: with branches here the sums would be moved about
    chunk(c, I0{});
    chunk(c + 1, I1{});
    chunk(c + 2, I2{});
    chunk(c + 3, I3{});
    c += 4;
  } while (c < nch);
  // no direct load may still be writing LDS; the last products are written before their sums are read
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int x = 0; x < 4; ++x) asm volatile("" : "+a"(acc[x][0]), "+a"(acc[x][1]), "+a"(acc[x][2]), "+a"(acc[x][3]));   // not before
  __builtin_amdgcn_sched_barrier(0);
  // the sums leave through LDS in whole rows, half of the wave's columns n at a time (see k_wgrad8)
  f4_t* const mine = reinterpret_cast<f4_t*>(lds) + wave * 2048;
  *reinterpret_cast<u32x4_t*>(&pattern[tid][0]) = pat[0];
  *reinterpret_cast<u32x4_t*>(&pattern[tid][16]) = pat[1];
  const int slot = lane & 31;
  const int64_t k = k0 + wk + 4 * slot;
  const bool inside = n0 + 256 <= N && k0 + 256 <= K;
#pragma unroll
  for (int y2 = 0; y2 < 2; ++y2) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const f16_t& c = acc[i >> 3][2 * y2 + ((i >> 2) & 1)];
      f4_t v = {c[4 * (i & 3)], c[4 * (i & 3) + 1], c[4 * (i & 3) + 2], c[4 * (i & 3) + 3]};
      if constexpr (DT == 0) v *= q8_pow2(127 + down[wave & 1]);
      mine[((lane & 31) + 32 * ((i >> 2) & 1)) * 32 + ((8 * (i >> 3) + 2 * (i & 3) + (lane >> 5)) ^ (lane & 31))] = v;
    }
    // Inside the matrix a store takes a few instructions: with one wave on a SIMD they are what the end of a tile costs
    // (rows of a step differ from the first's by a constant XOR and offset in LDS, by a uniform address in memory).
    if (inside && !meta) {
      const uint8_t* const t0 = reinterpret_cast<const uint8_t*>(mine);
      const uint32_t at = (uint32_t)(lane >> 5) * 512u + (uint32_t)((slot ^ (lane >> 5)) * 16);
      const uint32_t to = (uint32_t)(lane >> 5) * (uint32_t)K + 4u * slot;
      float* g = gW + (n0 + wn + 64 * y2) * K + k0 + wk;
#pragma unroll 1
      for (int u = 0; u < 4; ++u) {
        f4_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const f4_t*>(t0 + u * 8192 + j * 1024 + (at ^ (uint32_t)(((16 * u + 2 * j) & 31) * 16)));
#pragma unroll
        for (int j = 0; j < 8; ++j) __builtin_memcpy(g + (16 * u + 2 * j) * K + to, &v[j], 16);
      }
      continue;
    }
    if (inside) {
      // eight positions, four kept, a lane
      const uint8_t* const t0 = reinterpret_cast<const uint8_t*>(mine);
      const int r = lane >> 4, q = lane & 15;
      const uint32_t at = (uint32_t)r * 512u + (uint32_t)(((2 * q) ^ r) * 16);
      const uint32_t to = (uint32_t)r * (uint32_t)(K / 2) + 4u * q;
      const uint8_t* const pb = &pattern[wn + 64 * y2 + r][wk / 8 + q];
      float* g = gW + (n0 + wn + 64 * y2) * (K / 2) + (k0 + wk) / 2;
#pragma unroll 1
      for (int u = 0; u < 2; ++u) {
        uint32_t b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = pb[u * 1024 + j * 128];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint8_t* const t1 = t0 + u * 16384 + j * 2048;
          const uint32_t a0 = at ^ (uint32_t)(((4 * j) & 31) * 16), a1 = a0 ^ 16u;
          const f4_t o = {*reinterpret_cast<const float*>(t1 + (a0 | (b[j] & 3u) * 4)), *reinterpret_cast<const float*>(t1 + (a0 | (b[j] & 12u))),
                          *reinterpret_cast<const float*>(t1 + (a1 | ((b[j] >> 4) & 3u) * 4)), *reinterpret_cast<const float*>(t1 + (a1 | ((b[j] >> 4) & 12u)))};
          *reinterpret_cast<f4_t*>(g + (32 * u + 4 * j) * (K / 2) + to) = o;
        }
      }
      continue;
    }
    // (in a loop: written out, the stores of partial groups are more instructions than the products)
#pragma unroll 1
    for (int i = lane >> 5; i < 64; i += 16) {
      uint32_t byte[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) byte[j] = pattern[wn + 64 * y2 + i + 2 * j][(wk + 4 * slot) / 8];
      store_rows<8, 32>(gW, meta != nullptr, byte, mine, i, 2, n0 + wn + 64 * y2, N, slot, k, K);
    }
  }
#endif
}

// How a gradient is computed: 256 x 256 tiles (dY's rows aligned, if need be in a copy of them), or 128 x 128 tiles over
// `slices` slices of the rows.
struct GradPlan {
  bool wide, copy, narrow;
  int64_t slices, slice, slice_out;
  size_t off_part, bytes;   // workspace: the copied rows, the slices' sums from off_part on
};
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t x) { return (x + 255) & ~size_t(255); }

GradPlan grad_plan(int64_t M, int64_t N, int64_t K, bool masked, bool aligned) {
  GradPlan p{};
  // A wide tile's block stands alone on its CU, so its first loads and last stores show, and so do CUs left idle in the last
  // round of blocks; the small kernel has two on each. `use`: the share of the rounds' CUs that have a wide tile. us, wide
  // against small: 128 tiles of a possible 256, 2048 x 4096, M 4096 91 against 84; 160, 2560 x 4096, M 1024 35 against 40; 289 of
  // 512, 4100 x 4090, M 512 49 against 39; 304, 4096 x 4864, M 256 33 against 30, M 1024 68 both, M 4096 212 against 253; 897,
  // 9776 x 5786, M 64 57 against 53, M 96 60 both, M 192 71 against 84. At kept positions its stores are the shorter ones too:
  // 4096 x 4096, M 64 15 against 25.
  const int64_t wide = cdiv(N, 256) * cdiv(K, 256);
  const double use = (double)wide / (double)(cdiv(wide, 256) * 256);
  p.wide = M > 0 && use >= 0.58 && M >= (wide >= 256 && use >= 0.65 ? (masked ? 1 : 96) : 768) && N < (int64_t(1) << 22) - 16;
  p.copy = M > 0 && (p.wide ? !aligned : N < 16);        // (the other kernel takes pieces of 16)
  p.slices = 1;
  p.slice = M;
  if (p.copy) p.bytes = round256((size_t)M * (size_t)(cdiv(N, 16) * 16) * 2);
  if (p.wide) return p;
  const int64_t tiles = cdiv(N, 128) * cdiv(K, 128);
  // slices of at least 512 rows, so that their sums cost less than they save (999 x 2051 x 768: one slice 18.5 us, three
  // 19.9; 8192 x 128 x 128: sixteen 16.6, 32 19.2), up to a block a CU
  p.slices = std::max<int64_t>(1, std::min(256 / tiles, M / 512));
  p.slice = cdiv(cdiv(M, p.slices), 2 * kWM) * 2 * kWM;
  p.slices = std::max<int64_t>(1, cdiv(M, std::max<int64_t>(p.slice, 1)));
  // half as wide tiles on twice the CUs where the others would leave half of them idle (999 x 2051 x 768 14.4 us against 16.9,
  // 8192 x 256 x 256 in 16 slices 16.3 against 18.3; with every CU taken already 2048 x 2048 x 2048 34.0 against 31.0), but not
  // over few rows, where the more groups' sums cost more than that saves (100 x 300 x 300 8.5 against 6.8)
  p.narrow = tiles * p.slices <= 128 && M >= 512;
  p.slice_out = cdiv(N * (masked ? K / 2 : K), 64) * 64;
  p.off_part = p.bytes;
  if (p.slices > 1) p.bytes += (size_t)p.slices * (size_t)p.slice_out * 4;
  return p;
}

int check_grad(int64_t M, int64_t N, int64_t K, bool masked, bool aligned, GradPlan* p) {
  if (M < 0 || N < 1 || K < 1 || N > kMaxRow8 || K > kMaxRow8 || (masked && K % 16)) return SLIM_ESHAPE;
  if (cdiv(N, 128) * cdiv(K, 128) > 0x7FFFFFFF || M >= (int64_t(1) << 31) || M > ((int64_t(1) << 32) - 256) / cdiv(N, 16))      // (pieces of a copy are counted in 32 bits)
    return SLIM_EUNSUPPORTED;
  *p = grad_plan(M, N, K, masked, aligned);
  const bool fits = p->wide ? one_launch(8 * cdiv(cdiv(N, 256) * cdiv(K, 256), 8), 256)
                            : one_launch(cdiv(N, 128) * cdiv(K, p->narrow ? 64 : 128), 512);
  return fits ? SLIM_OK : SLIM_EUNSUPPORTED;
}

template <int DT>
int grad(const GradPlan& p, const uint16_t* dY, int64_t lddy, const uint8_t* xc, const uint8_t* xe, int64_t M, int64_t N, int64_t K,
         const uint8_t* meta, float* gW, void* ws, hipStream_t s) {
  int64_t cols = N;         // columns of dY's rows that may be read
  if (p.copy) {
    const int64_t pieces = cdiv(N, 16);
    uint16_t* rows = reinterpret_cast<uint16_t*>(ws);
    SlimKernelTimer timer("align_rows", s);
    SLIM_LAUNCH(timer, k_align_rows, dim3((unsigned)cdiv(M * pieces, 256)), dim3(256), s, dY, lddy, (uint32_t)N, (uint32_t)pieces,
                (uint32_t)(M * pieces), rows);
    dY = rows;
    cols = lddy = pieces * 16;
  }
  if (p.wide) {
    SlimKernelTimer timer("grad_w8_wide", s);
    SLIM_LAUNCH(timer, (k_wgrad8_wide<DT>), dim3((unsigned)(8 * cdiv(cdiv(N, 256) * cdiv(K, 256), 8))), dim3(256), s, dY, lddy, xc, xe,
                M, N, K, meta, gW);
    return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
  }
  const dim3 grid((unsigned)(cdiv(N, 128) * cdiv(K, p.narrow ? 64 : 128)), (unsigned)p.slices);
  float* out = p.slices > 1 ? reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + p.off_part) : gW;
  {
    SlimKernelTimer timer("grad_w8", s);
    if (p.narrow) SLIM_LAUNCH(timer, (k_wgrad8<DT, 64>), grid, dim3(512), s, dY, lddy, cols, xc, xe, M, N, K, meta, out, p.slice, p.slice_out);
    else SLIM_LAUNCH(timer, (k_wgrad8<DT, 128>), grid, dim3(512), s, dY, lddy, cols, xc, xe, M, N, K, meta, out, p.slice, p.slice_out);
  }
  if (p.slices > 1) {
    const int64_t count = N * (meta ? K / 2 : K);
    SlimKernelTimer timer("grad_w8_sum", s);
    SLIM_LAUNCH(timer, k_wgrad8_sum, dim3((unsigned)cdiv(count, 1024)), dim3(256), s, out, p.slices, p.slice_out, count, gW);
  }
  return hipGetLastError() == hipSuccess ? SLIM_OK : SLIM_EDEVICE;
}

// Rows that the wide kernel's direct loads take as they are.
bool aligned_rows(const void* dY, int64_t lddy) { return slim_aligned16(dY) && lddy % 8 == 0 && lddy < (int64_t(1) << 22); }

}  // namespace

extern "C" int slim_grad_w8_workspace(int64_t M, int64_t N, int64_t K, int masked, int aligned, size_t* bytes) {
  if (!bytes) return SLIM_EINVAL;
  GradPlan p;
  const int rc = check_grad(M, N, K, masked != 0, aligned != 0, &p);
  if (rc != SLIM_OK) return rc;
  *bytes = p.bytes;
  return SLIM_OK;
}

extern "C" int slim_grad_w8(const void* dY, int dtype, int64_t lddy, const uint8_t* xcodes, const uint8_t* xexps, int64_t M,
                            int64_t N, int64_t K, const uint8_t* meta, float* gW, void* ws, size_t ws_bytes, void* stream) {
  if (dtype != SLIM_F16 && dtype != SLIM_BF16) return SLIM_EDTYPE;
  GradPlan p;
  const int rc = check_grad(M, N, K, meta != nullptr, aligned_rows(dY, lddy), &p);
  if (rc != SLIM_OK) return rc;
  if (lddy < N) return SLIM_ESHAPE;
  if (!gW || (M > 0 && (!dY || !xcodes || !xexps))) return SLIM_EINVAL;
  if (!slim_aligned_to(dY, 2) || !slim_aligned16(xcodes) || !slim_aligned16(xexps) || !slim_aligned16(meta) ||
      !slim_aligned16(gW))
    return SLIM_EALIGN;
  if (p.bytes && (!ws || ws_bytes < p.bytes)) return SLIM_EWORKSPACE;
  if (p.bytes && !slim_aligned16(ws)) return SLIM_EALIGN;
  const uint16_t* y = reinterpret_cast<const uint16_t*>(dY);
  return dtype == SLIM_F16 ? grad<0>(p, y, lddy, xcodes, xexps, M, N, K, meta, gW, ws, (hipStream_t)stream)
                           : grad<1>(p, y, lddy, xcodes, xexps, M, N, K, meta, gW, ws, (hipStream_t)stream);
}
