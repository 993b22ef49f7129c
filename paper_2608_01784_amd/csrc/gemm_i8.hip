// SwiGLU experts and plain products on 8-bit integer rows and weights (int8.h): the launches of gemm8_impl.h.
//
// A row of the activation has one scale, so its codes wait for all of its columns: the up product leaves bf16 rows,
// which quantize_i8_kernel rounds to 8 bits ahead of the down product.
#include "gemm8_impl.h"

namespace rfx {
namespace {

const uint8_t* codes(const int8_t* p) { return reinterpret_cast<const uint8_t*>(p); }
const uint32_t* bits(const float* p) { return reinterpret_cast<const uint32_t*>(p); }

size_t act_bytes(int rows, int f) { return align_up(2 * static_cast<size_t>(rows) * f + 1); }
size_t code_bytes(int rows, int f) { return align_up(static_cast<size_t>(rows) * f + 1); }

}  // namespace

size_t swiglu_i8_ws_bytes(int rows, int f) {
  return act_bytes(rows, f) + code_bytes(rows, f) + align_up(sizeof(float) * (static_cast<size_t>(rows) + 1));
}

int launch_swiglu_i8(const int8_t* h, const float* hs, const int32_t* sorted_token, const int32_t* expert_offsets,
                     const Int8Weights& w, int T, int E, int d, int f, int cap, const AlwaysOnI8& sh, void* act,
                     uint16_t* y_sorted, hipStream_t s) {
  if (cap <= 0 && sh.rows <= 0) return REFLEX_OK;
  const int rows = cap + sh.rows;
  uint16_t* const a = static_cast<uint16_t*>(act);
  int8_t* const q = reinterpret_cast<int8_t*>(static_cast<char*>(act) + act_bytes(rows, f));
  float* const qs = reinterpret_cast<float*>(reinterpret_cast<char*>(q) + code_bytes(rows, f));
  const int likely = expected_rows(T, E, cap, sh.rows);
  const Args8 up{codes(h), bits(hs), sorted_token, expert_offsets, codes(w.w_gate), codes(w.w_up), bits(w.s_gate),
                 bits(w.s_up), codes(sh.w.w_gate), codes(sh.w.w_up), bits(sh.w.s_gate), bits(sh.w.s_up), E, d, f, T, cap,
                 sh.row0, sh.rows, nullptr, a, nullptr, 0};
  int rc = launch_gemm8<I8, UP, uint16_t>(up, likely, s);
  if (rc != REFLEX_OK) return rc;
  // (without routed experts the rows are the always-on expert's)
  rc = launch_quantize_i8(a, nullptr, E > 0 ? expert_offsets + E : nullptr, rows, rows, sh.rows > 0 ? sh.row0 : rows, f, q,
                          qs, s);
  if (rc != REFLEX_OK) return rc;
  const Args8 down{codes(q), bits(qs), nullptr, expert_offsets, codes(w.w_down), nullptr, bits(w.s_down), nullptr,
                   codes(sh.w.w_down), nullptr, bits(sh.w.s_down), nullptr, E, f, d, rows, cap, sh.row0, sh.rows, nullptr,
                   y_sorted, nullptr, 0};
  return launch_gemm8<I8, DOWN, uint16_t>(down, likely, s);
}

int launch_matmul_i8(const int8_t* x, const float* xs, const int8_t* w, const float* ws, const int32_t* n_rows, int M,
                     int N, int K, int out_type, void* out, hipStream_t s) {
  const Args8 a{codes(x), bits(xs), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, codes(w), nullptr, bits(ws), nullptr,
                0, K, N, M, M, 0, M, n_rows, out, nullptr, 0};
  return out_type == REFLEX_TYPE_F32 ? launch_gemm8<I8, PLAIN, float>(a, M, s) : launch_gemm8<I8, PLAIN, uint16_t>(a, M, s);
}

}  // namespace rfx
