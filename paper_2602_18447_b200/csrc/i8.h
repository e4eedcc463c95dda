// Host interface of the 8-bit integer kernels: rows to codes and back (rows_i8.cu), products of codes (gemm_i8.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace cs {

// Types of rows, as the C ABI numbers them.
constexpr int kF16 = 0, kBF16 = 1, kF32 = 2;
// The largest K whose sum of products of any two 8-bit codes fits 32 bits: 2^14 K < 2^31.
constexpr int kMaxI8K = 131056;
// Tokens and output channels of a product at most.
constexpr int kMaxI8Rows = 1 << 30;

struct QuantRows {
  const void* x;            // [rows, >= d] of `type`, rows x_stride elements apart
  const void* delta;        // the same of `delta_type`, or null
  void* x_out;              // x + delta, type of x; only with delta
  const float* gain;        // null: no norm
  int8_t* codes;            // [rows, d]
  float* scales;            // [rows]
  int64_t x_stride, delta_stride, x_out_stride;
  int32_t rows, d, type, delta_type;
  float eps;
};
// Rows to codes, the RMS norm in front of them where there are gains. d a multiple of 16; rows 16-byte aligned.
cudaError_t launch_quantize_i8(const QuantRows& p, cudaStream_t s);
// out [rows, d] of `type`, rows out_stride apart = codes * scale.
cudaError_t launch_dequantize_i8(const int8_t* codes, const float* scales, void* out, int64_t out_stride, int rows, int d, int type,
                                 cudaStream_t s);

struct GemmI8 {
  const int8_t *a, *w, *w2;                          // [M, K] rows a_stride apart, [N, K], [N, K] (gated) or null
  int64_t a_stride;
  const float *a_scales, *w_scales, *w2_scales;      // [M], [N], [N] (gated)
  const float* add;                                  // [M, >= N] or null
  void* out;                                         // [M, >= N] of `type` (kF32 only for ungated products, and with add)
  int64_t add_stride, out_stride;                    // elements
  int32_t M, N, K, type;
  int32_t weights_settled;      // nothing that may still run before this launch writes the weights
  uint32_t* status;             // null: the word that i8_status reads
};
// How a product reads its operands: boxes of so many rows of the activations (0: no maps) and of the weights, of one 128-byte piece
// of every row or of two (deep).
struct I8Box {
  int rows, w_rows;
  bool deep;
};
I8Box gemm_i8_box(int M, int N, int K, bool gated);
// Map over [rows, k] codes, rows `stride` bytes apart, 128-byte swizzle. k a multiple of 128 for deep boxes.
bool make_i8_map(CUtensorMap* tm, const int8_t* base, int rows, int k, int64_t stride, int box_rows, bool deep);
// out = the codes' product times both scales (+ add), or silu(first) * second. K a multiple of 16, at most kMaxI8K. Maps as gemm_i8_box
// says; tw2 is read for gated products only.
cudaError_t gemm_i8(const CUtensorMap& ta, const CUtensorMap& tw, const CUtensorMap& tw2, const GemmI8& p, cudaStream_t s);
// The time-out bits that launches without a status word of their own have left on this device, and clears them. Synchronises s.
cudaError_t i8_status(uint32_t* bits, cudaStream_t s);

}  // namespace cs
