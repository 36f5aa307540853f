// Device helpers shared by the kernels over the paged cache held in 4 bits (the format
// stands in heterofold.h).
#pragma once

#include "hf_attn.h"

namespace hf {

// Offsets in a head's part of a page.
template <int D>
struct PageHead {
  static constexpr int G = D / 32;
  int P;
  FI PageHead(int log2_page) : P(1 << log2_page) {}
  FI int bytes() const { return P * (D + 8 * G); }
  FI int kcode(int row) const { return row * (D / 2); }
  FI int vcode(int row) const { return P * (D / 2) + row * (D / 2); }  // row: of a block's first token
  FI int word(int role, int row) const { return P * D + (role * P + row) * (4 * G); }
};

FI float bf16_round(float x) { return (float)(__bf16)x; }

// Two codes of a dword, nibbles n and n + 4, as bf16 16 + code: moved to bits 3..6 of
// each half, under the exponent of 16.  The two constants are kept in registers
// (an instruction takes one literal at most), which makes a shift and one and-or of it.
struct Codes {
  uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
  FI Codes() { asm volatile("" : "+v"(mask), "+v"(sixteen)); }
  FI uint32_t two(uint32_t w, int n) const {
    return ((n == 0 ? w << 3 : w >> (4 * n - 3)) & mask) | sixteen;
  }
  // CENTRED: as code - 8, exact, for fp32: 16 + code beside sums of up to 16 would cost
  // four more bits of the fp32 accumulation than code - 8 does.
  template <bool CENTRED>
  FI bf16x8 operand(uint32_t w) const {
    union {
      uint32_t u[4];
      bf16x8 v;
    } x;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint32_t p = two(w, n);
      if (CENTRED) {
        const float lo = __builtin_bit_cast(float, p << 16) - 24.0f;
        const float hi = __builtin_bit_cast(float, p & 0xffff0000u) - 24.0f;
        x.u[n] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo),
                                       0x07060302u);  // (exact: the upper halves)
      } else {
        x.u[n] = p;
      }
    }
    return x.v;
  }
};

// x as S bf16 terms whose sum holds 8 S bits of it.
// (S = 1: x itself, which the conversion after it rounds.  So bf16 calls take a weight times
// its value's scale: three terms would take three times the second product's instructions, for
// an error the size of the result's own rounding, 2.3e-3 in all against 1.7e-3.)
template <int S>
FI void split(float x, float (&t)[S]) {
#pragma unroll
  for (int i = 0; i < S; ++i) {
    t[i] = S == 1 ? x : bf16_round(x);
    x -= t[i];
  }
}

template <int N>
FI void load_dwords(const uint8_t* p, uint32_t (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i + e] = v[e];
  }
}

}  // namespace hf
