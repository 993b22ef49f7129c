// 8-bit numbers with a scale for each block of 128 (e4m3 codes, power-of-two scales).
//
// A block's scale is s = 2^e with the smallest e for which its largest magnitude is at most
// 448 s (448: the largest e4m3 number), held as the byte e + 127.  Dividing by s is exact in
// fp32, so a code is its number rounded once (nearest, ties to even), and the matrix cores
// take the byte as it is (the scale operand of the f8f6f4 MFMA): no vector instruction is
// spent on scales between the products.  A power of two costs nothing in relative precision
// against an fp32 scale (e4m3 is itself floating point), only up to one of the 15 binades
// between the largest and the smallest normal number.
#pragma once

#include "common.h"

namespace rfx {

constexpr int F8_BLOCK = REFLEX_FP8_BLOCK;
constexpr uint32_t F8_ONE = 127;        // scale 1, of a block of zeros
constexpr uint32_t F8_MIN = 1;          // 2^-126: keeps 1 / s and s normal numbers

// Scale byte of a block from the bits of its largest magnitude (not negative, finite).
RFX_DEVICE uint32_t f8_scale_byte(uint32_t amax) {
  // amax = 1.m 2^(x - 127); 448 = 1.75 2^8
  const int e = static_cast<int>(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return amax == 0 ? F8_ONE : static_cast<uint32_t>(e < static_cast<int>(F8_MIN) ? static_cast<int>(F8_MIN) : e);
}

// 1 / s of a scale byte (1 .. 247).
RFX_DEVICE float f8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four e4m3 codes of four fp32 numbers within +-448.
RFX_DEVICE uint32_t f8_pack4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return static_cast<uint32_t>(v);
}

// Inclusive prefix sums of 64-bit numbers across a wave, as wave_inclusive_scan_i32 (lanes without a
// source add zero).
template <int CTRL, int ROWS, class T>
RFX_DEVICE T dpp_add64(T v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(u)), CTRL, ROWS, 0xf, false));
  const uint32_t hi = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(u >> 32)), CTRL, ROWS, 0xf, false));
  return v + __builtin_bit_cast(T, (static_cast<uint64_t>(hi) << 32) | lo);
}
template <class T>
RFX_DEVICE T wave_inclusive_scan64(T v) {
  static_assert(sizeof(T) == 8, "64-bit numbers");
  v = dpp_add64<0x111, 0xf>(v);      // row_shr:1, 2, 4, 8
  v = dpp_add64<0x112, 0xf>(v);
  v = dpp_add64<0x114, 0xf>(v);
  v = dpp_add64<0x118, 0xf>(v);
  v = dpp_add64<0x142, 0xa>(v);      // row_bcast:15 to rows 1, 3
  return dpp_add64<0x143, 0xc>(v);   // row_bcast:31 to rows 2, 3
}
// The sum over the wave, in every lane.
template <class T>
RFX_DEVICE T wave_sum64(T v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, wave_inclusive_scan64(v));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(u)), 63));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(u >> 32)), 63));
  return __builtin_bit_cast(T, (static_cast<uint64_t>(hi) << 32) | lo);
}

// Scales are kept in groups of four blocks (512 columns).
__host__ __device__ inline int f8_groups(int K) { return (K + 4 * F8_BLOCK - 1) / (4 * F8_BLOCK); }

// ---- launch wrappers (as in common.h) ---------------------------------------------------
size_t select_ws_bytes(int T);
int launch_select_rows(const uint8_t* masked, int T, int32_t* rows, int32_t* n_rows, void* ws, hipStream_t s);
int launch_quantize_rows(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, int x_rows, int M, int K,
                         uint8_t* q, uint8_t* scale, hipStream_t s);
int launch_quantize_weight(const uint16_t* w, int E, int N, int K, uint8_t* q, uint8_t* scale, hipStream_t s);

struct Fp8Weights {
  const uint8_t *w_gate, *w_up, *w_down, *s_gate, *s_up, *s_down;
};
struct AlwaysOn8 {      // as AlwaysOn
  Fp8Weights w;
  int row0, rows;
};
// Bytes of the 8-bit activation rows between the two products, codes and scales.
size_t swiglu8_ws_bytes(int rows, int f);
int launch_swiglu8_up(const uint8_t* h, const uint8_t* hs, const int32_t* sorted_token, const int32_t* expert_offsets,
                      const Fp8Weights& w, int T, int E, int d, int f, int cap, const AlwaysOn8& sh, uint8_t* act,
                      hipStream_t s);
int launch_swiglu8_down(const int32_t* expert_offsets, const Fp8Weights& w, int T, int E, int d, int f, int cap,
                        const AlwaysOn8& sh, const uint8_t* act, uint16_t* y_sorted, hipStream_t s);
int launch_swiglu8_dense(const uint8_t* x, const uint8_t* xs, const Fp8Weights& w, int M, int d, int f, uint16_t* y,
                         uint8_t* act, hipStream_t s);
int launch_matmul8(const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws, const int32_t* n_rows,
                   int M, int N, int K, int out_type, void* out, hipStream_t s);

size_t sample_ws_bytes(int M, int V);
int launch_sample(const void* logits, int logits_type, const int32_t* rows, const int32_t* n_rows, int M, int V,
                  const float* u, const reflex_sample_params& p, int T, int32_t* tokens, float* conf, void* ws,
                  hipStream_t s);

}  // namespace rfx
