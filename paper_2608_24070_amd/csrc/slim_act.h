// slim_act.h - activations and their derivatives in fp32, and what ends a row of a product or of a gradient with them.
#pragma once

#include <type_traits>

#include "slim.h"
#include "slim_q8.h"

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
// P of degree 8 fitted to erfcx(z) / (2 t) over z = 0 .. 9.5 for the least largest relative error (2e-8; 5e-7 in fp32), so
// that values far below zero keep their digits too.
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
    // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y)), y = sqrt(2 / pi) (x + 0.044715 x^3)
    const float y2 = x * __builtin_fmaf(0.0713548163f, x * x, 1.59576912f), p = act_rcp(1.f + act_exp(-y2));
    v = x * p;
    // past 12 the second term is below 2^-126 and its factors may pass fp32's range
    const float c = x > 12.f ? 12.f : x < -12.f ? -12.f : x;
    d = __builtin_fmaf(c * p * (1.f - p), __builtin_fmaf(0.214064449f, c * c, 1.59576912f), p);
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

// Ends rows eight columns a lane, 16 lanes for 128 columns of a row (all 16 take part in every call). DT: the type of 16-bit
// rows. Everything is fp32 until the one rounding of a result; a column's sum over rows takes du before it.
// A lane keeps the places of its columns in the first row; what is uniform is little then, for the tiles' scalar registers.
template <bool BWD, int DT>
struct ActRows {
  static constexpr bool kRows = true;
  static constexpr int kType = DT;
  ActArgs a;
  struct Lane {
    int n;               // columns that exist, 0 .. 8
    int place;           // of the eight in their group of 128 (0 .. 15), or -1 past the last group
    int tail;            // whether this lane writes one of the zeros behind the row's exponents: how far from its group's
    const char *p, *q;                 // u, mul or mul, res
    const uint8_t *pe, *qe;
    char *y, *w;
    uint8_t *ye, *we;
    float bias[8], s[8];
  };
  struct In {
    u32x4_t p, q;
    uint32_t pe, qe;
  };

  SLIM_DEV bool sums_wanted() const { return BWD && a.part; }
  SLIM_DEV void put_sum(int64_t block, int64_t col, int64_t N, float v) const { a.part[block * N + col] = v; }
  SLIM_DEV int code_row() const { return (int)q8_row(a.N); }
  SLIM_DEV int exp_row() const { return (int)q8_exp_row(a.N); }

  // Columns col .. col + 7 of rows from m0 on.
  SLIM_DEV void begin(Lane& l, int64_t m0, int64_t col) const {
    const int64_t left = a.N - col, g = col >> 7;
    l.n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    const bool in = col < code_row();
    l.place = in ? (int)(col >> 3) & 15 : -1;
    l.tail = in && g == (a.N - 1) >> 7 && l.place > 0 && l.place < 4 && g + l.place < exp_row() ? l.place : 0;
    const auto at = [&](const void* p, int64_t ld, bool q8) {
      return reinterpret_cast<const char*>(p) + (q8 ? m0 * code_row() + col : 2 * (m0 * ld + col));
    };
    const auto exp_at = [&](const uint8_t* e) { return e + m0 * exp_row() + g; };
    if constexpr (BWD) {
      l.p = at(a.u, a.ldu, a.q8);
      l.q = at(a.mul, a.ldmul, a.q8);
      l.pe = exp_at(a.ue);
      l.qe = exp_at(a.me);
    } else {
      l.p = at(a.mul, a.ldmul, false);
      l.q = at(a.res, a.ldres, false);
    }
    const bool y8 = !BWD && a.q8;
    l.y = const_cast<char*>(at(a.y, a.ldy, y8));
    l.w = const_cast<char*>(at(a.w, a.ldw, y8));
    l.ye = const_cast<uint8_t*>(exp_at(a.ye));
    l.we = const_cast<uint8_t*>(exp_at(a.we));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      l.s[e] = 0.f;
      l.bias[e] = 0.f;
      if constexpr (!BWD)
        if (a.bias && e < l.n) l.bias[e] = load_elem_rt(a.bias, col + e, a.bdt);
    }
  }

  // n, compared where it stands: the compiler keeps eight masks in scalar registers over the rows' loop otherwise
  static SLIM_DEV int here(int n) {
    asm volatile("" : "+v"(n));
    return n;
  }
  static SLIM_DEV u32x4_t load16(const char* p, int n) {
    u32x4_t v = {0, 0, 0, 0};
    if (n == 8) {
      __builtin_memcpy(&v, p, 16);
    } else {
      const uint16_t* t = reinterpret_cast<const uint16_t*>(p);
      const int k = here(n);
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < k) v[e >> 1] |= (uint32_t)t[e] << (16 * (e & 1));
    }
    return v;
  }
  // eight codes: those past the last column are there, and zero
  static SLIM_DEV u32x4_t load_codes(const char* p) {
    const u32x2_t v = *reinterpret_cast<const u32x2_t*>(p);
    return u32x4_t{v[0], v[1], 0, 0};
  }
  static SLIM_DEV void values(u32x4_t v, uint32_t b, bool q8, float* f) {
    if (q8) {
      q8_values4(v[0], q8_pow2(b), f);
      q8_values4(v[1], q8_pow2(b), f + 4);
    } else {
      act8_to_f(v, DT == 1, f);
    }
  }

  // What row m0 + row reads, if `ok`.
  SLIM_DEV void load(In& in, const Lane& l, int row, bool ok) const {
    in.p = in.q = u32x4_t{0, 0, 0, 0};
    in.pe = in.qe = 1;
    if (!ok || l.n == 0) return;
    if constexpr (BWD) {
      if (a.q8) {
        const int64_t c = (int64_t)row * code_row(), e = (int64_t)row * exp_row();
        if (a.u) {
          in.p = load_codes(l.p + c);
          in.pe = l.pe[e];
        }
        if (a.mul) {
          in.q = load_codes(l.q + c);
          in.qe = l.qe[e];
        }
      } else {
        if (a.u) in.p = load16(l.p + 2 * row * a.ldu, l.n);
        if (a.mul) in.q = load16(l.q + 2 * row * a.ldmul, l.n);
      }
    } else {
      if (a.mul) in.p = load16(l.p + 2 * row * a.ldmul, l.n);
      if (a.res) in.q = load16(l.q + 2 * row * a.ldres, l.n);
    }
  }

  SLIM_DEV void store_codes(char* p, uint8_t* ep, int row, const Lane& l, bool ok, const float* f) const {
    float v[8];
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = e < l.n ? f[e] : 0.f;
      big = max(big, q8_abs(v[e]));
    }
    const uint32_t b = q8_exponent(row16_max_u32(big));
    if (!ok || l.place < 0) return;
    const float s = q8_inverse(b);
    *reinterpret_cast<u32x2_t*>(p + (int64_t)row * code_row()) =
        u32x2_t{q8_codes4(v[0], v[1], v[2], v[3], s), q8_codes4(v[4], v[5], v[6], v[7], s)};
    uint8_t* const e = ep + (int64_t)row * exp_row();
    if (l.place == 0 || l.tail) e[l.tail] = l.tail ? 0 : (uint8_t)b;      // the row's last word ends in zeros
  }

  // Ends row m0 + row, whose sums are f.
  SLIM_DEV void eight(Lane& l, const In& in, int row, bool ok, float* f) const {
    float y[8], w[8];
    if constexpr (BWD) {
      float u[8];
      values(in.p, in.pe, a.q8, u);
      with_act(a.act, [&](auto A) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v, d;
          act_both<decltype(A)::value>(u[e], v, d);
          y[e] = f[e] * d;
          w[e] = f[e] * v;
        }
      });
      if (a.mul) {
        values(in.q, in.qe, a.q8, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= u[e];
      }
      if (a.part)
#pragma unroll
        for (int e = 0; e < 8; ++e) l.s[e] += ok ? y[e] : 0.f;      // of columns past the last: not asked for
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = f[e] + l.bias[e];
      with_act(a.act, [&](auto A) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = act_value<decltype(A)::value>(w[e]);
      });
      float o[8];
      if (a.mul) {
        act8_to_f(in.p, DT == 1, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= o[e];
      }
      if (a.res) {
        act8_to_f(in.q, DT == 1, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += o[e];
      }
      if (a.q8) {
        store_codes(l.y, l.ye, row, l, ok, y);
        if (a.w) store_codes(l.w, l.we, row, l, ok, w);
        return;
      }
    }
    if (ok && l.n) {
      const int n = l.n == 8 ? 8 : here(l.n);
      store8<DT>(l.y + 2 * row * a.ldy, 0, n, y);
      if (a.w) store8<DT>(l.w + 2 * row * a.ldw, 0, n, w);
    }
  }

  // Forward, 16 bits: four columns of a row, `left` of them.
  SLIM_DEV void four(int64_t m, int64_t n, int64_t left, f4_t v) const {
    static_assert(!BWD);
    float z[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = v[e] + (a.bias && e < left ? load_elem_rt(a.bias, n + e, a.bdt) : 0.f);
    with_act(a.act, [&](auto A) {
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
