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

// Eight consecutive values of a row as they are held, and as fp32.
template <int TYPE>
struct Piece {
  uint32_t w[TYPE == kF32 ? 8 : 4];
};
template <int TYPE>
__device__ __forceinline__ Piece<TYPE> load_piece(const void* row, int unit) {
  Piece<TYPE> p;
  constexpr int n = TYPE == kF32 ? 2 : 1;
  const uint4* from = static_cast<const uint4*>(row) + n * unit;
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const uint4 a = from[i];
    p.w[4 * i] = a.x; p.w[4 * i + 1] = a.y; p.w[4 * i + 2] = a.z; p.w[4 * i + 3] = a.w;
  }
  return p;
}
template <int TYPE>
__device__ __forceinline__ void store_piece(void* row, int unit, const Piece<TYPE>& p) {
  constexpr int n = TYPE == kF32 ? 2 : 1;
  uint4* to = static_cast<uint4*>(row) + n * unit;
#pragma unroll
  for (int i = 0; i < n; ++i) to[i] = make_uint4(p.w[4 * i], p.w[4 * i + 1], p.w[4 * i + 2], p.w[4 * i + 3]);
}
template <int TYPE>
__device__ __forceinline__ void values(const Piece<TYPE>& p, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = TYPE == kF32   ? make_float2(__uint_as_float(p.w[(TYPE == kF32 ? 2 : 1) * j]), __uint_as_float(p.w[TYPE == kF32 ? 2 * j + 1 : j]))
                     : TYPE == kF16 ? unpack_f16x2(p.w[j])
                                    : make_float2(bf16_lo(p.w[j]), bf16_hi(p.w[j]));
    v[2 * j] = f.x;
    v[2 * j + 1] = f.y;
  }
}
template <int TYPE>
__device__ __forceinline__ Piece<TYPE> held(const float (&v)[8]) {
  Piece<TYPE> p;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (TYPE == kF32) {
      p.w[(TYPE == kF32 ? 2 : 1) * j] = __float_as_uint(v[2 * j]);
      p.w[TYPE == kF32 ? 2 * j + 1 : j] = __float_as_uint(v[2 * j + 1]);
    } else {
      p.w[j] = TYPE == kF16 ? pack_f16x2(v[2 * j], v[2 * j + 1]) : pack_bf16x2(v[2 * j], v[2 * j + 1]);
    }
  }
  return p;
}

// Eight codes. 1.5 * 2^23 added in the same rounding as the product leaves the nearest integer in the low bits of the sum. The
// product y * inv is off the quotient by at most 127 * 2^-24, the rounding of inv, so a remainder that is not within 2^-16 of a half
// decides the code. For the others the sign of 127 y - (c + 1/2) most is taken exactly: both products as a rounded part and its error.
// (One value in thirty thousand, but in 16-bit rows half of the largest magnitude, a tie, is met in every few hundred.)
__device__ __forceinline__ uint2 codes8(const float (&y)[8], float inv, float most) {
  constexpr float kMagic = 12582912.0f, kNear = 0.5f - 0x1p-16f;
  float t[8], rem[8], worst = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    t[j] = fmaf(y[j], inv, kMagic);
    rem[j] = fmaf(y[j], inv, -(t[j] - kMagic));
    worst = fmaxf(worst, fabsf(rem[j]));
  }
  if (worst > kNear) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float half = t[j] - kMagic + copysignf(0.5f, rem[j]);
      const float p = __fmul_rn(127.0f, y[j]), q = __fmul_rn(half, most);
      const float d = (p - q) + (fmaf(127.0f, y[j], -p) - fmaf(half, most, -q));
      const float c = d > 0.f ? half + 0.5f : d < 0.f ? half - 0.5f : rintf(half);
      if (fabsf(rem[j]) > kNear) t[j] = c + kMagic;
    }
  }
  uint2 r;
  r.x = __byte_perm(__byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040),
                    __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040), 0x5410);
  r.y = __byte_perm(__byte_perm(__float_as_uint(t[4]), __float_as_uint(t[5]), 0x0040),
                    __byte_perm(__float_as_uint(t[6]), __float_as_uint(t[7]), 0x0040), 0x5410);
  return r;
}

struct RowStats {
  uint32_t most;     // bits of the largest magnitude: ordered as the magnitudes are, infinity and NaN above all numbers
  float squares;
};
// Over the threads of a row, the same order every time.
template <bool NORM>
__device__ __forceinline__ RowStats row_stats(RowStats s, RowStats* shared) {
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

// blockDim.x threads to a row; several rows to a block (blockDim.y) only where a row has one warp. DELTA < 0: nothing is added. A
// thread holds NV pieces of eight values, as they came, between the row's statistics and its codes; a longer row is read again.
// What counts is how many rows an SM has on their way: registers are kept to 32 a thread where the types allow it.
template <int TYPE, int DELTA, bool NORM, int NV>
__global__ void __launch_bounds__(1024, TYPE == kF32 || NORM || NV > 2 ? 1 : 2) quantize_i8_kernel(const QuantRows p) {
  __shared__ RowStats shared[32];
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kBytes = TYPE == kF32 ? 4 : 2, kDeltaBytes = DELTA == kF32 ? 4 : 2;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (row >= p.rows) return;
  const void* x = static_cast<const uint8_t*>(p.x) + row * p.x_stride * kBytes;
  const void* delta = DELTA < 0 ? nullptr : static_cast<const uint8_t*>(p.delta) + row * p.delta_stride * kDeltaBytes;
  void* x_out = DELTA < 0 ? nullptr : static_cast<uint8_t*>(p.x_out) + row * p.x_out_stride * kBytes;
  const int units = p.d >> 3;

  RowStats s = {0u, 0.f};
  const auto add = [&](int unit, Piece<TYPE> a, const Piece<(DELTA < 0 ? kF16 : DELTA)>& b) {
    if (DELTA < 0) return a;
    float v[8], w[8];
    values<TYPE>(a, v);
    values<(DELTA < 0 ? kF16 : DELTA)>(b, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += w[j];
    a = held<TYPE>(v);
    store_piece<TYPE>(x_out, unit, a);
    return a;
  };
  const auto gained = [&](int unit, float (&v)[8]) {
    if (!NORM) return;
    float g[8];
    values<kF32>(load_piece<kF32>(p.gain, unit), g);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= g[j];
  };
  const auto look = [&](int unit, const Piece<TYPE>& a) {
    float v[8];
    values<TYPE>(a, v);
    if (NORM) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s.squares = fmaf(v[j], v[j], s.squares);
    }
    gained(unit, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s.most = max(s.most, __float_as_uint(v[j]) & 0x7fffffffu);
  };

  Piece<TYPE> held_x[NV];
  Piece<(DELTA < 0 ? kF16 : DELTA)> held_d[DELTA < 0 ? 1 : NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int unit = threadIdx.x + i * blockDim.x;
    if (unit < units) {
      held_x[i] = load_piece<TYPE>(x, unit);
      if (DELTA >= 0) held_d[DELTA < 0 ? 0 : i] = load_piece<(DELTA < 0 ? kF16 : DELTA)>(delta, unit);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int unit = threadIdx.x + i * blockDim.x;
    if (unit < units) {
      held_x[i] = add(unit, held_x[i], held_d[DELTA < 0 ? 0 : i]);
      look(unit, held_x[i]);
    }
  }
  for (int unit = threadIdx.x + NV * blockDim.x; unit < units; unit += blockDim.x)
    look(unit, add(unit, load_piece<TYPE>(x, unit), DELTA < 0 ? held_d[0] : load_piece<(DELTA < 0 ? kF16 : DELTA)>(delta, unit)));
  s = row_stats<NORM>(s, shared);

  const float most = __uint_as_float(s.most);
  bool good = s.most < 0x7f800000u;
  float scale = most / 127.0f;
  if (NORM) {
    good = good && s.squares < __uint_as_float(0x7f800000u);
    scale = most > 0.f ? most / sqrtf(s.squares / static_cast<float>(p.d) + p.eps) / 127.0f : 0.f;
  }
  if (threadIdx.x == 0) p.scales[row] = good ? scale : __uint_as_float(0x7fffffffu);
  // Rows far from 1 are brought nearer, by a power of two, so that neither inv nor a product leaves the normal range; values that this
  // makes subnormal have codes of 0 either way.
  const float by = most < 0x1p-60f ? 0x1p90f : most > 0x1p100f ? 0x1p-60f : 1.0f;
  const float top = most * by, inv = 127.0f / top;
  const bool any = good && most > 0.f;
  uint2* codes = reinterpret_cast<uint2*>(p.codes + row * p.d);
  const auto put = [&](int unit, const Piece<TYPE>& a) {
    float v[8];
    values<TYPE>(a, v);
    gained(unit, v);
    if (by != 1.0f) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= by;
    }
    codes[unit] = any ? codes8(v, inv, top) : make_uint2(0u, 0u);
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int unit = threadIdx.x + i * blockDim.x;
    if (unit < units) put(unit, held_x[i]);
  }
  for (int unit = threadIdx.x + NV * blockDim.x; unit < units; unit += blockDim.x)
    put(unit, load_piece<TYPE>(DELTA < 0 ? x : x_out, unit));          // what this thread stored above
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
    store_piece<TYPE>(static_cast<uint8_t*>(out) + row * out_stride * kBytes, unit, held<TYPE>(v));
  }
}

template <int TYPE, int DELTA, bool NORM>
cudaError_t launch_rows(const QuantRows& p, cudaStream_t s) {
  const int units = p.d >> 3;
  const int nv = (p.rows <= kNumSMs && units <= 1024) ? 1 : units <= 2048 ? 2 : 4;
  const int threads = std::min(1024, (units + 32 * nv - 1) / (32 * nv) * 32), together = threads == 32 ? 8 : 1;
  const auto kernel = nv == 1   ? quantize_i8_kernel<TYPE, DELTA, NORM, 1>
                      : nv == 2 ? quantize_i8_kernel<TYPE, DELTA, NORM, 2>
                                : quantize_i8_kernel<TYPE, DELTA, NORM, 4>;
  const cudaError_t e = launch_pdl(kernel, dim3((p.rows + together - 1) / together), dim3(threads, together), 0, s, p);
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
