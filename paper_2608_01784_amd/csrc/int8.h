// 8-bit integers with a scale for each row (a token of the input, an output channel of the weights).
//
// a = the row's largest magnitude (2^-100 at least), s = a / 127, a code is rint(x (127 / a)): each operation
// rounded to fp32 once, ties to even, so |code| <= 127.  A product of two rows is s t times a sum of integers, which
// is exact in 32 bits (K <= 16384: |sum| <= 2^28), in any order: results do not depend on tiles or splits.
#pragma once

#include "fp8.h"

namespace rfx {

constexpr uint32_t I8_LEAST = 0x0d800000u;      // 2^-100: s and 127 / a are normal numbers
constexpr uint32_t I8_INF = 0x7f800000u;

// A product and a sum rounded to fp32 by themselves (the compiler would join them to one rounding otherwise).
RFX_DEVICE float mul_rn(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
RFX_DEVICE float add_rn(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

// From the bits of a row's largest magnitude: its scale (NaN where the row is not finite) and what its numbers are
// multiplied by (0 there: codes 0).
RFX_DEVICE float i8_scale(uint32_t amax) {
  return amax >= I8_INF ? __uint_as_float(0x7fc00000u) : __uint_as_float(max(amax, I8_LEAST)) / 127.0f;
}
RFX_DEVICE float i8_factor(uint32_t amax) {
  return amax >= I8_INF ? 0.0f : 127.0f / __uint_as_float(max(amax, I8_LEAST));
}

// Four codes of two packed bf16 pairs.  1.5 2^23 added, a number of magnitude below 2^22 is rounded to an integer
// (nearest, ties to even) whose two's complement is the sum's low bits.  (A row that is not finite has factor 0 and
// may hold 0 times infinity: its codes are masked.)
RFX_DEVICE uint32_t i8_pack4(uint32_t ab, uint32_t cd, float factor) {
  auto code = [factor](uint32_t bits) {
    return __float_as_uint(add_rn(mul_rn(__uint_as_float(bits), factor), 12582912.0f));
  };
  const uint32_t a = code(ab << 16), b = code(ab & 0xffff0000u), c = code(cd << 16), d = code(cd & 0xffff0000u);
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
  return factor == 0.0f ? 0u : lo | hi;
}

// Largest magnitude of eight bf16 numbers, as fp32 bits (infinities and NaN above all others).
RFX_DEVICE uint32_t i8_amax8(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max((w[i] << 16) & 0x7fffffffu, w[i] & 0x7fff0000u));
  return m;
}

// ---- launch wrappers (as in common.h) ---------------------------------------------------
// rows, n_rows as in reflex_quantize_int8; rows from `extra` on are quantised whatever n_rows says (extra = M: none).
int launch_quantize_i8(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, size_t x_rows, size_t M,
                       size_t extra, int K, int8_t* q, float* scale, hipStream_t s);

struct Int8Weights {
  const int8_t *w_gate, *w_up, *w_down;
  const float *s_gate, *s_up, *s_down;
};
struct AlwaysOnI8 {      // as AlwaysOn
  Int8Weights w;
  int row0, rows;
};
// Bytes of the activation rows between the two products: bf16, then codes, then scales.
size_t swiglu_i8_ws_bytes(int rows, int f);
int launch_swiglu_i8(const int8_t* h, const float* hs, const int32_t* sorted_token, const int32_t* expert_offsets,
                     const Int8Weights& w, int T, int E, int d, int f, int cap, const AlwaysOnI8& sh, void* act,
                     uint16_t* y_sorted, hipStream_t s);
int launch_matmul_i8(const int8_t* x, const float* xs, const int8_t* w, const float* ws, const int32_t* n_rows, int M,
                     int N, int K, int out_type, void* out, hipStream_t s);

int launch_block_norm(const reflex_norm_args& a, hipStream_t s);

}  // namespace rfx
