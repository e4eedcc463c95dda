// Rows to 8-bit codes with one scale each, the RMS norm in front of them, and codes back to values.
//
// A row y has A = max |y|, the scale A / 127 and the codes rint(127 y / A), ties to even, of the quotient as a real number. The
// norm's row is y = x g / rms(x): its factor 1 / rms is common to y and A, so that it drops out of the codes; they are taken from
// fp32(x g), and only the scale carries the factor. A row that holds a NaN or an infinity gets codes of 0 and the scale NaN.
//
// Bound by memory: a row is read once, held in registers while its maximum (and the sum of its squares) is formed, and written.
#include "i8.h"

#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace cs {

namespace {

// Eight consecutive values of a row as fp32.
template <int TYPE>
__device__ __forceinline__ void load8(const void* row, int unit, float (&v)[8]) {
  if (TYPE == kF32) {
    const float4* p = static_cast<const float4*>(row) + 2 * unit;
    const float4 a = p[0], b = p[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 a = static_cast<const uint4*>(row)[unit];
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = TYPE == kF16 ? unpack_f16x2(w[j]) : make_float2(bf16_lo(w[j]), bf16_hi(w[j]));
      v[2 * j] = f.x;
      v[2 * j + 1] = f.y;
    }
  }
}
// The other way; v is left as the values that were stored.
template <int TYPE>
__device__ __forceinline__ void store8(void* row, int unit, float (&v)[8]) {
  if (TYPE == kF32) {
    float4* p = static_cast<float4*>(row) + 2 * unit;
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = TYPE == kF16 ? pack_f16x2(v[2 * j], v[2 * j + 1]) : pack_bf16x2(v[2 * j], v[2 * j + 1]);
      const float2 f = TYPE == kF16 ? unpack_f16x2(w[j]) : make_float2(bf16_lo(w[j]), bf16_hi(w[j]));
      v[2 * j] = f.x;
      v[2 * j + 1] = f.y;
    }
    static_cast<uint4*>(row)[unit] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Eight codes. 1.5 * 2^23 added in the same rounding as the product leaves the nearest integer in the low bits of the sum. The
// product y * inv is off the quotient by at most 127 * 2^-24, the rounding of inv, so a remainder that is not within 2^-16 of a half
// decides the code; the others (one in thirty thousand) take the quotient in 64 bits, whose rounding cannot cross a half that 24-bit
// operands do not lie on.
__device__ __forceinline__ uint2 codes8(const float (&y)[8], float inv, float most) {
  constexpr float kMagic = 12582912.0f;
  uint32_t b[8];
  float worst = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float t = fmaf(y[j], inv, kMagic);
    worst = fmaxf(worst, fabsf(fmaf(y[j], inv, -(t - kMagic))));
    b[j] = __float_as_uint(t);
  }
  if (worst > 0.5f - 0x1p-16f || inv > 0x1p126f) {      // the latter: a largest magnitude so small that inv may be infinite
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
      float yj = y[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) yj = j == i ? y[i] : yj;
      const uint32_t c = static_cast<uint32_t>(__double2int_rn(127.0 * static_cast<double>(yj) / static_cast<double>(most)));
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = j == i ? c : b[i];
    }
  }
  uint2 r;
  r.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  r.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
  return r;
}

struct RowStats {
  uint32_t most;     // bits of the largest magnitude: ordered as the magnitudes are, infinity and NaN above all numbers
  float squares;
};
// Over all threads of the block, the same order every time.
template <bool NORM>
__device__ __forceinline__ RowStats block_stats(RowStats s, RowStats* shared) {
  s.most = __reduce_max_sync(0xffffffffu, s.most);
  if (NORM) s.squares = warp_sum(s.squares);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return s;
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = s;
  __syncthreads();
  s = (threadIdx.x & 31) < warps ? shared[threadIdx.x & 31] : RowStats{0u, 0.f};
  s.most = __reduce_max_sync(0xffffffffu, s.most);
  if (NORM) s.squares = warp_sum(s.squares);
  return s;
}

// One block per row. DELTA < 0: nothing is added. A thread holds up to NV pieces of eight values; a longer row is read again.
template <int TYPE, int DELTA, bool NORM, int NV>
__global__ void __launch_bounds__(1024) quantize_i8_kernel(const QuantRows p) {
  __shared__ RowStats shared[32];
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kBytes = TYPE == kF32 ? 4 : 2, kDeltaBytes = DELTA == kF32 ? 4 : 2;
  const int64_t row = blockIdx.x;
  const void* x = static_cast<const uint8_t*>(p.x) + row * p.x_stride * kBytes;
  const void* delta = DELTA < 0 ? nullptr : static_cast<const uint8_t*>(p.delta) + row * p.delta_stride * kDeltaBytes;
  void* x_out = DELTA < 0 ? nullptr : static_cast<uint8_t*>(p.x_out) + row * p.x_out_stride * kBytes;
  const int units = p.d >> 3;

  RowStats s = {0u, 0.f};
  const auto take = [&](int unit, const void* from, bool add, float (&v)[8]) {
    load8<TYPE>(from, unit, v);
    if (DELTA >= 0 && add) {
      float w[8];
      load8<(DELTA < 0 ? kF16 : DELTA)>(delta, unit, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += w[j];
      store8<TYPE>(x_out, unit, v);
    }
  };
  const auto gained = [&](int unit, float (&v)[8]) {
    if (!NORM) return;
    float g[8];
    load8<kF32>(p.gain, unit, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= g[j];
  };
  const auto look = [&](int unit, float (&v)[8]) {
    if (NORM) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s.squares = fmaf(v[j], v[j], s.squares);
    }
    gained(unit, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s.most = max(s.most, __float_as_uint(v[j]) & 0x7fffffffu);
  };

  float y[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int unit = threadIdx.x + i * blockDim.x;
    if (unit < units) {
      take(unit, x, true, y[i]);
      look(unit, y[i]);
    }
  }
  for (int unit = threadIdx.x + NV * blockDim.x; unit < units; unit += blockDim.x) {
    float v[8];
    take(unit, x, true, v);
    look(unit, v);
  }
  s = block_stats<NORM>(s, shared);

  const float most = __uint_as_float(s.most);
  bool good = s.most < 0x7f800000u;
  float scale = most / 127.0f;
  if (NORM) {
    good = good && s.squares < __uint_as_float(0x7f800000u);
    scale = most > 0.f ? most / sqrtf(s.squares / static_cast<float>(p.d) + p.eps) / 127.0f : 0.f;
  }
  if (threadIdx.x == 0) p.scales[row] = good ? scale : __uint_as_float(0x7fffffffu);
  const float inv = 127.0f / most;
  uint2* codes = reinterpret_cast<uint2*>(p.codes + row * p.d);
  const bool any = good && most > 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int unit = threadIdx.x + i * blockDim.x;
    if (unit < units) codes[unit] = any ? codes8(y[i], inv, most) : make_uint2(0u, 0u);
  }
  for (int unit = threadIdx.x + NV * blockDim.x; unit < units; unit += blockDim.x) {
    float v[8];
    take(unit, DELTA < 0 ? x : x_out, false, v);      // what this thread stored above
    gained(unit, v);
    codes[unit] = any ? codes8(v, inv, most) : make_uint2(0u, 0u);
  }
}

template <int TYPE>
__global__ void dequantize_i8_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales, void* __restrict__ out,
                                     int64_t out_stride, int rows, int d) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kBytes = TYPE == kF32 ? 4 : 2;
  const int64_t units = d >> 3, all = units * rows;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t row = i / units;
    const int unit = static_cast<int>(i - row * units);
    const uint2 c = reinterpret_cast<const uint2*>(codes)[i];
    const float s = scales[row];
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = s * static_cast<float>(static_cast<int8_t>((j < 4 ? c.x : c.y) >> (8 * (j & 3))));
    store8<TYPE>(static_cast<uint8_t*>(out) + row * out_stride * kBytes, unit, v);
  }
}

template <int TYPE, int DELTA, bool NORM>
cudaError_t launch_rows(const QuantRows& p, cudaStream_t s) {
  const int threads = std::min(1024, ((p.d >> 3) + 127) / 128 * 32);
  const cudaError_t e = launch_pdl(quantize_i8_kernel<TYPE, DELTA, NORM, 4>, dim3(p.rows), dim3(threads), 0, s, p);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantize_i8(const QuantRows& p, cudaStream_t s) {
  if (p.rows <= 0) return cudaSuccess;
  if (!p.gain) {
    switch (p.type) {
      case kF16: return launch_rows<kF16, -1, false>(p, s);
      case kBF16: return launch_rows<kBF16, -1, false>(p, s);
      default: return launch_rows<kF32, -1, false>(p, s);
    }
  }
  switch (p.type) {
    case kF16: return p.delta ? launch_rows<kF16, kF16, true>(p, s) : launch_rows<kF16, -1, true>(p, s);
    case kBF16: return p.delta ? launch_rows<kBF16, kBF16, true>(p, s) : launch_rows<kBF16, -1, true>(p, s);
    default:
      if (!p.delta) return launch_rows<kF32, -1, true>(p, s);
      return p.delta_type == kF16    ? launch_rows<kF32, kF16, true>(p, s)
             : p.delta_type == kBF16 ? launch_rows<kF32, kBF16, true>(p, s)
                                     : launch_rows<kF32, kF32, true>(p, s);
  }
}

cudaError_t launch_dequantize_i8(const int8_t* codes, const float* scales, void* out, int64_t out_stride, int rows, int d, int type,
                                 cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  const int64_t blocks = (static_cast<int64_t>(d >> 3) * rows + 255) / 256;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(blocks, kNumSMs * 8)));
  const auto kernel = type == kF16 ? dequantize_i8_kernel<kF16> : type == kBF16 ? dequantize_i8_kernel<kBF16> : dequantize_i8_kernel<kF32>;
  const cudaError_t e = launch_pdl(kernel, grid, dim3(256), 0, s, codes, scales, out, out_stride, rows, d);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace cs
