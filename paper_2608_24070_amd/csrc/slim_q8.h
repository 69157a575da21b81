// slim_q8.h - device helpers of the 8-bit path: e4m3 codes with one power of two per group of 128.
#pragma once

#include "slim_device.h"

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f2_t __attribute__((ext_vector_type(2)));

// Most columns of a row kept in 8 bits (256 rows stay within 32-bit byte offsets), most groups of one operand, and most that
// one launch of eight lanes a group takes (a launch holds fewer than 2^32 threads).
constexpr int64_t kMaxRow8 = int64_t(1) << 22;
constexpr int64_t kMaxGroups8 = (int64_t(1) << 32) - 64;
constexpr int64_t kMaxQuant8 = (int64_t(1) << 29) - 64;

// Whether one launch takes so many blocks side by side: it holds fewer than 2^32 threads.
constexpr bool one_launch(int64_t blocks, int64_t threads) { return blocks < (int64_t(1) << 32) / threads; }

// Fitted sizes: codes per row (whole groups) and exponent bytes per row (whole 32-bit words).
constexpr int64_t q8_row(int64_t k) { return (k + 127) / 128 * 128; }
constexpr int64_t q8_exp_row(int64_t k) { return (k + 511) / 512 * 4; }

// Biased exponent b = e + 127 of a group whose largest finite magnitude has fp32 bits `amax`: e is the smallest integer
// with amax / 2^e <= 448 = 1.75 * 2^8, that is floor(log2 amax) - 8, and one more where the mantissa passes 1.75 (the
// addend carries into the exponent field exactly then). At least 1 (e = -126), so that 2^-e is a normal fp32 number; at
// most 247. Powers of two cost no accuracy against a scale of amax / 448: e4m3 values keep their relative precision,
// and the products with 2^e and 2^-e are exact.
SLIM_DEV uint32_t q8_exponent(uint32_t amax) {
  const int b = (int)((amax + 0x1FFFFFu) >> 23) - 8;
  return (uint32_t)(b > 1 ? b : 1);
}
SLIM_DEV float q8_pow2(uint32_t b) { return __builtin_bit_cast(float, b << 23); }              // 2^(b - 127)
SLIM_DEV float q8_inverse(uint32_t b) { return __builtin_bit_cast(float, (254u - b) << 23); }  // 2^(127 - b)

// |x| as fp32 bits for a group's maximum; a NaN or an infinity counts as zero there (its own code is NaN).
SLIM_DEV uint32_t q8_abs(float x) {
  const uint32_t a = abs_bits(x);
  return a < 0x7F800000u ? a : 0u;
}

// Four values times s (a power of two) as e4m3 codes: round to nearest, ties to even; NaN and infinities give NaN.
SLIM_DEV uint32_t q8_codes4(float a, float b, float c, float d, float s) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * s, b * s, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * s, d * s, v, true);
}

// Element types by the codes of slim_dtype: 0 fp16, 1 bf16, 2 fp32.
template <int DT> constexpr int elem_bytes() { return DT == 2 ? 4 : 2; }

template <int DT>
SLIM_DEV float load_elem(const void* p, int64_t i) {
  if constexpr (DT == 2) return reinterpret_cast<const float*>(p)[i];
  else if constexpr (DT == 1) return __builtin_bit_cast(float, (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
  else return (float)reinterpret_cast<const _Float16*>(p)[i];
}
SLIM_DEV float load_elem_rt(const void* p, int64_t i, int dt) {
  return dt == 2 ? load_elem<2>(p, i) : dt == 1 ? load_elem<1>(p, i) : load_elem<0>(p, i);
}

// fp32 -> 16 bits, nearest, ties to even (NaN stays NaN)
SLIM_DEV uint32_t to_bf16(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x); }
SLIM_DEV uint32_t to_f16(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x); }
template <int DT>
SLIM_DEV uint32_t to_16(float x) { return DT == 1 ? to_bf16(x) : to_f16(x); }

template <int DT>
SLIM_DEV void store_elem(void* p, int64_t i, float x) {
  if constexpr (DT == 2) reinterpret_cast<float*>(p)[i] = x;
  else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)to_16<DT>(x);
}

// Eight consecutive elements from i on, of which the first `n` exist (the others read as zero, and no byte past the
// n-th element is touched). Rows may start at any element: 16-byte global accesses need no alignment here.
template <int DT>
SLIM_DEV void load8(const void* p, int64_t i, int64_t n, float* f) {
  if (n >= 8) {
    const char* q = reinterpret_cast<const char*>(p) + i * elem_bytes<DT>();
    if constexpr (DT == 2) {
      f4_t a, b;
      __builtin_memcpy(&a, q, 16);
      __builtin_memcpy(&b, q + 16, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = a[e];
        f[4 + e] = b[e];
      }
    } else {
      u32x4_t v;
      __builtin_memcpy(&v, q, 16);
      act8_to_f(v, DT == 1, f);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = e < n ? load_elem<DT>(p, i + e) : 0.f;
  }
}

template <int DT>
SLIM_DEV void store8(void* p, int64_t i, int64_t n, const float* f) {
  if (n >= 8) {
    char* q = reinterpret_cast<char*>(p) + i * elem_bytes<DT>();
    if constexpr (DT == 2) {
      const f4_t a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
      __builtin_memcpy(q, &a, 16);
      __builtin_memcpy(q + 16, &b, 16);
    } else {
      u32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = to_16<DT>(f[2 * e]) | (to_16<DT>(f[2 * e + 1]) << 16);
      __builtin_memcpy(q, &v, 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) store_elem<DT>(p, i + e, f[e]);
  }
}

// Four e4m3 codes times s as fp32 (exact)
SLIM_DEV void q8_values4(uint32_t c, float s, float* f) {
  const f2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  f[0] = lo[0] * s;
  f[1] = lo[1] * s;
  f[2] = hi[0] * s;
  f[3] = hi[1] * s;
}

// Largest value over aligned groups of 8 lanes, given to each of them: swaps of neighbours, of pairs and, mirrored, of
// the two quads (DPP quad_perm 1 0 3 2, quad_perm 2 3 0 1, row_half_mirror).
SLIM_DEV uint32_t oct_max_u32(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));
}
