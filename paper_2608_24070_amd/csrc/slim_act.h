// slim_act.h - activations and their derivatives in fp32, and what ends a row of a product or of a gradient with them.
#pragma once

#include <type_traits>

#include "slim.h"
#include "slim_q8.h"

// A lambda that is always inlined: one that is not keeps what it refers to in memory.
#define SLIM_INLINE __attribute__((always_inline))

// f(integral_constant A) for the activation `act` (uniform)
template <class F>
SLIM_DEV void with_act(int act, F&& f) {
  switch (act) {
    case SLIM_ACT_RELU: return f(std::integral_constant<int, SLIM_ACT_RELU>{});
    case SLIM_ACT_GELU: return f(std::integral_constant<int, SLIM_ACT_GELU>{});
    case SLIM_ACT_GELU_TANH: return f(std::integral_constant<int, SLIM_ACT_GELU_TANH>{});
    case SLIM_ACT_SILU: return f(std::integral_constant<int, SLIM_ACT_SILU>{});
    default: return f(std::integral_constant<int, SLIM_ACT_NONE>{});
  }
}

// e^x and 1 / x to one unit in the last place, and e^x's of its argument's rounding (x log2 e, 2^-24 |x|): a value of 24 bits where
// its result leaves in 16 or 8.
SLIM_DEV float act_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
SLIM_DEV float act_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// Phi(x), the normal distribution, and e = exp(-x^2 / 2). Its tail erfc(|x| / sqrt 2) / 2 is e t P(t), t = 1 / (1 + 0.3 |x| / sqrt 2),
// P of degree 8 fitted to erfcx(z) / (2 t) over z = 0 .. 9.5 for the least largest relative error (4e-8 with these constants, 5e-7 in fp32),
// so that values far below zero keep their digits too: with e's rounding of its argument the tail is 1e-6 off at |x| = 4, 8e-6 at 13.
SLIM_DEV float act_phi(float x, float& e) {
  const float t = act_rcp(__builtin_fmaf(0.212132034f, __builtin_fabsf(x), 1.f));
  e = act_exp(-0.5f * x * x);
  constexpr float c[9] = {0.0845948085f, 0.0853459686f, 0.0742412210f, 0.107218117f, -0.0468155667f, 0.273197442f, -0.255613148f, 0.242548183f,
                          -0.0647170320f};
  float p = c[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) p = __builtin_fmaf(p, t, c[i]);
  const float tail = e * (p * t);
  return x < 0.f ? tail : 1.f - tail;
}

// v = act(x), d = act'(x); what is not used costs nothing.
template <int A>
SLIM_DEV void act_both(float x, float& v, float& d) {
  if constexpr (A == SLIM_ACT_RELU) {
    v = x < 0.f ? 0.f : x;            // a NaN stays one
    d = x > 0.f ? 1.f : 0.f;
  } else if constexpr (A == SLIM_ACT_GELU) {
    float e;
    const float phi = act_phi(x, e);
    v = x * phi;
    d = __builtin_fmaf(x * 0.398942280f, e, phi);
  } else if constexpr (A == SLIM_ACT_GELU_TANH) {
    // (1 + tanh y) / 2 = 1 / (1 + 2^(-2 y log2 e)), y = sqrt(2 / pi) (x + 0.044715 x^3); past 12 that is 0 or 1 to fp32, and the slope's
    // second term nothing, so x^2 may stop there and stays in range
    const float c = __builtin_amdgcn_fmed3f(x, -12.f, 12.f), c2 = c * c;
    const float p = act_rcp(1.f + __builtin_amdgcn_exp2f(x * __builtin_fmaf(-0.102943240f, c2, -2.30220819f)));
    v = x * p;
    d = __builtin_fmaf(c * __builtin_fmaf(-p, p, p), __builtin_fmaf(0.214064449f, c2, 1.59576912f), p);
  } else if constexpr (A == SLIM_ACT_SILU) {
    const float p = act_rcp(1.f + act_exp(-x));
    v = x * p;
    d = __builtin_fmaf(v, 1.f - p, p);
  } else {
    v = x;
    d = 1.f;
  }
}
template <int A>
SLIM_DEV float act_value(float x) {
  float v, d;
  act_both<A>(x, v, d);
  return v;
}

// Largest value over aligned groups of 16 lanes, given to each of them (DPP row_ror 1, 2, 4, 8).
SLIM_DEV uint32_t row16_max_u32(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
}

// Global memory by name: a pointer whose origin the compiler does not see would be a flat one, which takes the LDS's counter too.
#define SLIM_GLOBAL __attribute__((address_space(1)))
typedef u32x4_t u32x4_any_t __attribute__((aligned(2)));

// What a row's end reads and writes. Forward: z = sums + bias, y = act(z) mul + res, w = z. Backward: y = du = dh mul act'(u),
// w = dmul = dh act(u). N columns; rows in 8 bits have q8_row(N) codes and q8_exp_row(N) exponents.
struct ActArgs {
  int act, bdt;
  int q8;                                                       // forward: y and w leave in 8 bits; backward: u and mul are 8-bit rows
  int64_t N;
  const void* bias;                                             // forward, or null
  const void* u; const uint8_t* ue; int64_t ldu;                // backward
  const void* mul; const uint8_t* me; int64_t ldmul;            // or null
  const uint16_t* res; int64_t ldres;                           // forward, or null
  void* y; uint8_t* ye; int64_t ldy;
  void* w; uint8_t* we; int64_t ldw;                            // or null
  float* part;                                                  // backward: sums of y over each block's rows [blocks][N], or null
};

// Ends rows eight columns a lane, 16 lanes for 128 columns of a row (all 16 take part in every call), and some rows at a time, `step`
// apart: their reads, an activation's chains of dependent steps and the choices that are the launch's go side by side. DT: the type of
// 16-bit rows. Everything is fp32 until the one rounding of a result; a column's sum over rows takes du before it.
// A lane keeps its places in what is read and in what is written, and the ways to the next row, in vector registers: the tiles' scalar
// ones are few.
template <bool BWD, int DT>
struct ActRows {
  static constexpr bool kRows = true;
  static constexpr int kType = DT;
  ActArgs a;
  struct Lane {
    int n;                             // columns that exist, 0 .. 8
    int place;                         // of the eight in their group of 128 (0 .. 15), or -1 past the last group
    int tail;                          // whether this lane writes one of the zeros behind the row's exponents: how far from its group's
    const char *p, *q;                 // u, mul or mul, res: the next row to read
    const uint8_t *pe, *qe;
    char *y, *w;                       // the next row to write
    uint8_t *ye, *we;
    int64_t p_by, q_by, y_by, w_by;
    int e_by;
    float bias[8], s[8];
  };
  struct In {
    u32x4_t p, q;
    uint32_t pe, qe;
  };
  // what there is to do (one scalar)
  enum { kQ8 = 1, kP = 2, kQ = 4, kW = 8, kBias = 16, kSums = 32 };
  SLIM_DEV int todo() const {
    return (a.q8 ? kQ8 : 0) | ((BWD ? a.u : a.mul) ? kP : 0) | ((BWD ? a.mul != nullptr : a.res != nullptr) ? kQ : 0) | (a.w ? kW : 0) |
           (a.bias ? kBias : 0) | (a.part ? kSums : 0);
  }

  SLIM_DEV bool sums_wanted() const { return BWD && a.part; }
  SLIM_DEV void put_sum(int64_t block, int64_t col, int64_t N, float v) const { ((SLIM_GLOBAL float*)a.part)[block * N + col] = v; }

  template <class T>
  static SLIM_DEV T in_vector(T v) {
    asm volatile("" : "+v"(v));
    return v;
  }

  // Columns col .. col + 7 of rows m, m + step, ...
  SLIM_DEV void begin(Lane& l, int64_t m, int step, int64_t col) const {
    const int64_t left = a.N - col, g = col >> 7, codes = q8_row(a.N), exps = q8_exp_row(a.N);
    l.n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    const bool in = col < codes;
    l.place = in ? (int)(col >> 3) & 15 : -1;
    l.tail = in && g == (a.N - 1) >> 7 && l.place > 0 && l.place < 4 && g + l.place < exps ? l.place : 0;
    const bool in8 = BWD && a.q8, out8 = !BWD && a.q8;
    const auto at = [&](const void* p, int64_t ld, bool q8) { return reinterpret_cast<const char*>(p) + (q8 ? m * codes + col : 2 * (m * ld + col)); };
    const auto by = [&](int64_t ld, bool q8) { return in_vector((q8 ? codes : 2 * ld) * step); };
    const auto exp_at = [&](const uint8_t* e) { return e + m * exps + g; };
    const int64_t ldp = BWD ? a.ldu : a.ldmul, ldq = BWD ? a.ldmul : a.ldres;
    l.p = at(BWD ? a.u : a.mul, ldp, in8);
    l.q = at(BWD ? a.mul : a.res, ldq, in8);
    l.pe = exp_at(a.ue);
    l.qe = exp_at(a.me);
    l.y = const_cast<char*>(at(a.y, a.ldy, out8));
    l.w = const_cast<char*>(at(a.w, a.ldw, out8));
    l.ye = const_cast<uint8_t*>(exp_at(a.ye)) + l.tail;
    l.we = const_cast<uint8_t*>(exp_at(a.we)) + l.tail;
    l.p_by = by(ldp, in8);
    l.q_by = by(ldq, in8);
    l.y_by = by(a.ldy, out8);
    l.w_by = by(a.ldw, out8);
    l.e_by = in_vector((int)exps * step);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      l.s[e] = 0.f;
      l.bias[e] = 0.f;
      if constexpr (!BWD)
        if (a.bias && e < l.n) l.bias[e] = load_elem_rt(a.bias, col + e, a.bdt);
    }
  }

  // n, compared where it stands: the compiler keeps eight masks in scalar registers over the rows' loop otherwise
  static SLIM_DEV int here(int n) { return in_vector(n); }
  static SLIM_DEV u32x4_t load16(const char* p, int n) {
    u32x4_t v = {0, 0, 0, 0};
    if (n == 8) {
      v = *(const SLIM_GLOBAL u32x4_any_t*)p;
    } else {
      const SLIM_GLOBAL uint16_t* t = (const SLIM_GLOBAL uint16_t*)p;
      const int k = here(n);
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < k) v[e >> 1] |= (uint32_t)t[e] << (16 * (e & 1));
    }
    return v;
  }
  // eight codes: those past the last column are there, and zero
  static SLIM_DEV u32x4_t load_codes(const char* p) {
    const u32x2_t v = *(const SLIM_GLOBAL u32x2_t*)p;
    return u32x4_t{v[0], v[1], 0, 0};
  }
  static SLIM_DEV void values(u32x4_t v, uint32_t b, bool q8, float* f) {
    if (q8) {
      // (the instruction scales: a multiplication a value less than q8_values4, whose values these are down to 2^-126)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f2_t t = i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v[i >> 1], q8_pow2(b), true)
                             : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v[i >> 1], q8_pow2(b), false);
        f[2 * i] = t[0];
        f[2 * i + 1] = t[1];
      }
    } else {
      act8_to_f(v, DT == 1, f);
    }
  }

  // The next NB rows of this lane, of which those `step` b < more are there (WHOLE: all of them and all columns): what they read.
  template <bool WHOLE, int NB = 4>
  SLIM_DEV void load_rows(In* in, Lane& l, int todo, int step, int more) const {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      in[b].p = in[b].q = u32x4_t{0, 0, 0, 0};
      in[b].pe = in[b].qe = 1;
    }
    const auto there = [&](int b) { return WHOLE || (step * b < more && l.n > 0); };
    if (todo & kP) {
#pragma unroll
      for (int b = 0; b < NB; ++b, l.p += l.p_by) {
        if (BWD && (todo & kQ8)) {
          if (there(b)) {
            in[b].p = load_codes(l.p);
            in[b].pe = *(const SLIM_GLOBAL uint8_t*)l.pe;
          }
          l.pe += l.e_by;
        } else if (there(b)) {
          in[b].p = load16(l.p, WHOLE ? 8 : l.n);
        }
      }
    }
    if (todo & kQ) {
#pragma unroll
      for (int b = 0; b < NB; ++b, l.q += l.q_by) {
        if (BWD && (todo & kQ8)) {
          if (there(b)) {
            in[b].q = load_codes(l.q);
            in[b].qe = *(const SLIM_GLOBAL uint8_t*)l.qe;
          }
          l.qe += l.e_by;
        } else if (there(b)) {
          in[b].q = load16(l.q, WHOLE ? 8 : l.n);
        }
      }
    }
  }

  // The largest finite magnitude's bits of eight values. A NaN loses every comparison of v_max3_f32, whose operands' signs cost
  // nothing: half an instruction a value, where q8_abs and a maximum take four. An infinity wins; then they are gone through again.
  static SLIM_DEV uint32_t largest(const float* v) {
    float m = 0.f;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int e = 0; e < 8; e += 2) asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(m) : "v"(v[e]), "v"(v[e + 1]));
#endif
    uint32_t big = abs_bits(m);
    if (__ballot(big >= 0x7F800000u)) {
      big = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) big = max(big, q8_abs(v[e]));
    }
    return big;
  }
  template <bool WHOLE, int NB>
  static SLIM_DEV void store_codes(char*& p, uint8_t*& ep, int64_t by, const Lane& l, int step, int more, const float (*f)[8]) {
#pragma unroll
    for (int b = 0; b < NB; ++b, p += by, ep += l.e_by) {
      float v[8];
      const int n = WHOLE ? 8 : here(l.n);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = WHOLE || e < n ? f[b][e] : 0.f;
      const uint32_t x = q8_exponent(row16_max_u32(largest(v)));
      if (!WHOLE && (step * b >= more || l.place < 0)) continue;
      const float s = q8_inverse(x);
      *(SLIM_GLOBAL u32x2_t*)p = u32x2_t{q8_codes4(v[0], v[1], v[2], v[3], s), q8_codes4(v[4], v[5], v[6], v[7], s)};
      if (l.place == 0 || l.tail) *(SLIM_GLOBAL uint8_t*)ep = l.tail ? 0 : (uint8_t)x;      // the row's last word ends in zeros
    }
  }
  template <bool WHOLE>
  static SLIM_DEV void store_row(char* at, const Lane& l, bool there, const float* f) {
    if (!WHOLE && !(there && l.n)) return;
    u32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_16<DT>(f[2 * e]) | (to_16<DT>(f[2 * e + 1]) << 16);
    if (WHOLE || l.n == 8) {
      *(SLIM_GLOBAL u32x4_any_t*)at = v;
    } else {
      const int n = here(l.n);
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < n) ((SLIM_GLOBAL uint16_t*)at)[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
    }
  }
  template <bool WHOLE, int NB>
  static SLIM_DEV void store_rows(char*& p, int64_t by, const Lane& l, int step, int more, const float (*f)[8]) {
#pragma unroll
    for (int b = 0; b < NB; ++b, p += by) store_row<WHOLE>(p, l, step * b < more, f[b]);
  }

  // Ends the next NB rows, whose sums are f.
  template <bool WHOLE, int NB = 4>
  SLIM_DEV void end_rows(Lane& l, const In* in, int todo, int step, int more, float (*f)[8]) const {
    if constexpr (BWD) {
      with_act(a.act, [&](auto A) SLIM_INLINE {
        const auto rows = [&](auto gated) SLIM_INLINE {
#pragma unroll
          for (int b = 0; b < NB; ++b, l.y += l.y_by) {
            const bool there = WHOLE || step * b < more;
            float u[8], m[8], o[8];
            values(in[b].p, in[b].pe, todo & kQ8, u);
            if constexpr (decltype(gated)::value) values(in[b].q, in[b].qe, todo & kQ8, m);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float v, d;
              act_both<decltype(A)::value>(u[e], v, d);
              o[e] = f[b][e] * v;
              f[b][e] *= d;
              if constexpr (decltype(gated)::value) f[b][e] *= m[e];
            }
            if (todo & kSums)
#pragma unroll
              for (int e = 0; e < 8; ++e) l.s[e] += there ? f[b][e] : 0.f;      // of columns past the last: not asked for
            store_row<WHOLE>(l.y, l, there, f[b]);
            if constexpr (decltype(gated)::value) {
              store_row<WHOLE>(l.w, l, there, o);
              l.w += l.w_by;
            }
          }
        };
        if (todo & kQ) rows(std::true_type{});
        else rows(std::false_type{});
      });
    } else {
      if (todo & kBias)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 8; ++e) f[b][e] += l.bias[e];
      if (todo & kW) {
        if (todo & kQ8) store_codes<WHOLE, NB>(l.w, l.we, l.w_by, l, step, more, f);
        else store_rows<WHOLE, NB>(l.w, l.w_by, l, step, more, f);
      }
      with_act(a.act, [&](auto A) SLIM_INLINE {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 8; ++e) f[b][e] = act_value<decltype(A)::value>(f[b][e]);
      });
      float o[8];
      if (todo & kP)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          act8_to_f(in[b].p, DT == 1, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[b][e] *= o[e];
        }
      if (todo & kQ)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          act8_to_f(in[b].q, DT == 1, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[b][e] += o[e];
        }
      if (todo & kQ8) store_codes<WHOLE, NB>(l.y, l.ye, l.y_by, l, step, more, f);
      else store_rows<WHOLE, NB>(l.y, l.y_by, l, step, more, f);
    }
  }

  // Forward, 16 bits: four columns of a row, `left` of them.
  SLIM_DEV void four(int64_t m, int64_t n, int64_t left, f4_t v) const {
    static_assert(!BWD);
    float z[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = v[e] + (a.bias && e < left ? load_elem_rt(a.bias, n + e, a.bdt) : 0.f);
    with_act(a.act, [&](auto A) SLIM_INLINE {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = act_value<decltype(A)::value>(z[e]);
    });
    const auto read = [&](const void* p, int64_t at, float* o) {
      u32x2_t t = {0, 0};
      const uint16_t* s = reinterpret_cast<const uint16_t*>(p) + at;
      if (left >= 4) {
        __builtin_memcpy(&t, s, 8);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < left) t[e >> 1] |= (uint32_t)s[e] << (16 * (e & 1));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = act_to_f(t[e >> 1] >> (16 * (e & 1)) & 0xFFFFu, DT == 1);
    };
    float o[4];
    if (a.mul) {
      read(a.mul, m * a.ldmul + n, o);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= o[e];
    }
    if (a.res) {
      read(a.res, m * a.ldres + n, o);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += o[e];
    }
    const auto write = [&](void* p, int64_t at, const float* o4) {
      uint16_t* t = reinterpret_cast<uint16_t*>(p) + at;
      if (left >= 4) {
        const u32x2_t b = {to_16<DT>(o4[0]) | to_16<DT>(o4[1]) << 16, to_16<DT>(o4[2]) | to_16<DT>(o4[3]) << 16};
        __builtin_memcpy(t, &b, 8);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < left) t[e] = (uint16_t)to_16<DT>(o4[e]);
      }
    };
    write(a.y, m * a.ldy + n, y);
    if (a.w) write(a.w, m * a.ldw + n, z);
  }
};
