// Rows to 8-bit codes with one scale each, the RMS norm in front of them, codes back to values, and the rotary turn of rows that a
// product of codes has left.
//
// A row y has A = max |y|, the scale A / 127 and the codes rint(127 y / A), ties to even, of the quotient as a real number. The
// norm's row is y = x g / rms(x): its factor 1 / rms is common to y and A, so that it drops out of the codes; they are taken from
// fp32(x g), and only the scale carries the factor. A row that holds a NaN or an infinity gets codes of 0 and the scale NaN.
//
// Bound by memory: a row is read once, held in registers while its maximum (and the sum of its squares) is formed, and written.
// 5377 x 8960 bf16: 28.7 us, 5.0 TB/s of reads and writes, and 26.5 us, 5.5 TB/s, back again; norm and residual of 8191 x 3584 bf16:
// 36.1 us, 5.7 TB/s; of one row of 1536: 1.9 us, a round trip to memory and the two exchanges over the block.
#include "i8.h"

#include <algorithm>

#include "common.cuh"
#include "gemm.h"
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

// Numbers a little above and below 127 / most.
struct Inverse {
  float up, down, most;
};
__device__ __forceinline__ Inverse inverse_of(float most) {
  const uint32_t near = __float_as_uint(__fdividef(127.0f, most));      // off by two steps at most
  return {__uint_as_float(near + 3), __uint_as_float(near - 3), most};
}
__device__ __forceinline__ uint2 low_bytes(const uint32_t (&b)[8]) {
  uint2 r;
  r.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  r.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
  return r;
}
// Eight codes. 1.5 * 2^23 added in the same rounding as the product leaves the nearest integer in the low bits of the sum. Where the
// two inverses give one integer, it is the quotient's. Else the half between the two is compared with the quotient exactly: the sign
// of 127 y - half * most, both products as a rounded part and its error. (One value in twenty thousand; in 16-bit rows half of the
// largest magnitude, a tie, is met in every few hundred.)
__device__ __forceinline__ uint2 codes8(const float (&y)[8], const Inverse& by) {
  constexpr float kMagic = 12582912.0f;
  uint32_t b[8], differ = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    b[j] = __float_as_uint(fmaf(y[j], by.up, kMagic));
    differ |= b[j] ^ __float_as_uint(fmaf(y[j], by.down, kMagic));
  }
  if (differ) {
    uint32_t which = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) which |= b[j] != __float_as_uint(fmaf(y[j], by.down, kMagic)) ? 1u << j : 0u;
#pragma unroll 1
    for (; which; which &= which - 1) {
      const int at = __ffs(which) - 1;
      float v = y[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) v = at == j ? y[j] : v;
      const float half = 0.5f * ((fmaf(v, by.up, kMagic) - kMagic) + (fmaf(v, by.down, kMagic) - kMagic));
      const float p = __fmul_rn(127.0f, v), q = __fmul_rn(half, by.most);
      const float d = (p - q) + (fmaf(127.0f, v, -p) - fmaf(half, by.most, -q));
      const float c = d > 0.f ? half + 0.5f : d < 0.f ? half - 0.5f : rintf(half);
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = at == j ? __float_as_uint(c + kMagic) : b[j];
    }
  }
  return low_bytes(b);
}
// Eight codes of a row that came in 16 bits. Let y have the significand m < 2^11. 127 y / A is a tie, or it is off the next one by
// 1 / (254 m) > 2^-19 of itself at least, as 254 y - (2 k + 1) A is a whole number of units of y's last place; `up` is off by five
// steps at most, 5 * 2^-23. So one product decides all but the ties. Of those, A / 2 goes to 64, as its product with `up` does; others
// need a significand of A that 127, a prime, divides (`ties`; one row in 128). Without the second product and without A / 2, which two
// warps' pieces in five hold, among the doubtful 5377 x 8960 bf16 takes 33.6 -> 28.9 us.
__device__ __forceinline__ uint2 codes8_of_16_bits(const float (&y)[8], const Inverse& by, bool ties) {
  if (ties) return codes8(y, by);
  uint32_t b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = __float_as_uint(fmaf(y[j], by.up, 12582912.0f));
  return low_bytes(b);
}
// The larger of m and |v|; NaN if either is.
__device__ __forceinline__ float larger(float m, float v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(v)));
  return r;
}

struct RowStats {
  float most;        // the largest magnitude, NaN where a value is
  float squares;
};
// Over the threads of a row, the same order every time.
template <bool NORM>
__device__ __forceinline__ RowStats row_stats(RowStats s, RowStats* shared) {
  s.most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(s.most)));       // ordered as the bits are, NaN above all
  if (NORM) s.squares = warp_sum(s.squares);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return s;
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = s;
  __syncthreads();
  s = (threadIdx.x & 31) < warps ? shared[threadIdx.x & 31] : RowStats{0.f, 0.f};
  s.most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(s.most)));       // ordered as the bits are, NaN above all
  if (NORM) s.squares = warp_sum(s.squares);
  return s;
}

// blockDim.x threads to a row; several rows to a block (blockDim.y) only where a row has one warp. DELTA < 0: nothing is added. A
// thread holds NV pieces of eight values, as they came, between the row's statistics and its codes; a longer row is read again.
// What counts is how many rows an SM has on their way: registers are kept to 32 a thread where the types allow it.
template <int TYPE, int DELTA, bool NORM, int NV>
__global__ void __launch_bounds__(NV == 4 ? 640 : 1024, NV == 4 && TYPE != kF32 ? 2 : 1) quantize_i8_kernel(const QuantRows p) {
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

  RowStats s = {0.f, 0.f};
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
  uint32_t most2 = 0;       // 16-bit rows without gains: the magnitudes' bits, two at a time
  const auto look = [&](int unit, const Piece<TYPE>& a) {
    if (!NORM && TYPE != kF32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) most2 = __vmaxu2(most2, a.w[j] & 0x7fff7fffu);
      return;
    }
    float v[8];
    values<TYPE>(a, v);
    if (NORM) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s.squares = fmaf(v[j], v[j], s.squares);
    }
    gained(unit, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s.most = larger(s.most, v[j]);
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
  if (!NORM && TYPE != kF32) {
    const uint32_t m = max(most2 >> 16, most2 & 0xffffu);
    s.most = TYPE == kF16 ? __half2float(__ushort_as_half(static_cast<uint16_t>(m))) : __uint_as_float(m << 16);
  }
  s = row_stats<NORM>(s, shared);

  const float most = s.most;
  bool good = most < __uint_as_float(0x7f800000u);
  // the squares' mean has to be a normal number, or eps to stand in for it
  if (NORM) good = good && s.squares < __uint_as_float(0x7f800000u) && (s.squares >= p.d * 0x1p-126f || p.eps > 0.f || most == 0.f);
  if (threadIdx.x == 0) {
    float scale = most / 127.0f;
    if (NORM && most > 0.f) scale = most / sqrtf(s.squares / static_cast<float>(p.d) + p.eps) / 127.0f;
    p.scales[row] = good ? scale : __uint_as_float(0x7fffffffu);
  }
  // Rows far from 1 are brought nearer, by a power of two, so that neither inv nor a product leaves the normal range; values that this
  // makes subnormal have codes of 0 either way.
  const float by = most < 0x1p-60f ? 0x1p90f : most > 0x1p100f ? 0x1p-60f : 1.0f;
  const Inverse inverse = inverse_of(most * by);
  const bool any = good && most > 0.f;
  const bool ties = ((__float_as_uint(inverse.most) & 0x7fffffu) | 0x800000u) % 127u == 0;
  uint2* codes = reinterpret_cast<uint2*>(p.codes + row * p.d);
  const auto put = [&](int unit, const Piece<TYPE>& a) {
    float v[8];
    values<TYPE>(a, v);
    gained(unit, v);
    if (by != 1.0f) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= by;
    }
    uint2 c = make_uint2(0u, 0u);
    if (any) c = !NORM && TYPE != kF32 ? codes8_of_16_bits(v, inverse, ties) : codes8(v, inverse);
    codes[unit] = c;
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int unit = threadIdx.x + i * blockDim.x;
    if (unit < units) put(unit, held_x[i]);
  }
  for (int unit = threadIdx.x + NV * blockDim.x; unit < units; unit += blockDim.x)
    put(unit, load_piece<TYPE>(DELTA < 0 ? x : x_out, unit));          // what this thread stored above
}

// A thread per 16 codes. Bound by memory, 5377 x 8960 bf16 26.5 us, 5.4 TB/s. A byte with its sign turned, put under the exponent of 2^23, is 2^23 + 128 + code.
template <int TYPE>
__global__ void __launch_bounds__(256) dequantize_i8_kernel(const int8_t* codes, const float* scales, void* out, int64_t out_stride,
                                                            int rows, int d) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kBytes = TYPE == kF32 ? 4 : 2;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (row >= rows) return;
  const float s = scales[row];
  const uint4* from = reinterpret_cast<const uint4*>(codes + row * d);
  void* to = static_cast<uint8_t*>(out) + row * out_stride * kBytes;
  for (int unit = threadIdx.x + blockIdx.y * blockDim.x; unit < d >> 4; unit += blockDim.x * gridDim.y) {
    const uint4 c = from[unit];
    const uint32_t w[4] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u, c.z ^ 0x80808080u, c.w ^ 0x80808080u};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = s * (__uint_as_float(__byte_perm(w[2 * h + (j >> 2)], 0x4b000000u, 0x7540 + (j & 3))) - 8388736.0f);
      store_piece<TYPE>(to, 2 * unit + h, held<TYPE>(v));
    }
  }
}

// Rotary turn of projected rows in place, behind the 8-bit projection. A thread has the same four pairs of kRopeHeads heads of a token,
// so that it reads their angles once. Memory from L2, where the projection has left it; bound by latency (1163 tokens x 14 heads of
// 128: 7.2 us between two events, some 3 of them the events'; a warp to a head and two-byte accesses 8.7).
constexpr int kRopeHeads = 2;
template <int HALF>
__global__ void __launch_bounds__(256) rope_rows_kernel(__half* rows, int row_elems, int T, const RopeEpilogue rope) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kLanes = HALF / 4;                       // of a head
  const int heads = rope.n_rot_cols / (2 * HALF), groups = (heads + kRopeHeads - 1) / kRopeHeads;
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) / kLanes;
  const int lane = threadIdx.x % kLanes;
  const int t = static_cast<int>(i / groups), head0 = static_cast<int>(i - static_cast<int64_t>(t) * groups) * kRopeHeads;
  const bool here = t < T;                               // whole heads of lanes at a time; the others take part in the sums below
  __half* at = rows + static_cast<int64_t>(t) * row_elems + lane * 4;
  const float4* table = reinterpret_cast<const float4*>(rope.table + static_cast<int64_t>(t) * HALF + lane * 4);
  uint2 ra[kRopeHeads] = {}, rb[kRopeHeads] = {};
  float4 cs[2] = {};
#pragma unroll
  for (int h = 0; h < kRopeHeads; ++h) {
    if (here && head0 + h < heads) {
      ra[h] = *reinterpret_cast<const uint2*>(at + (head0 + h) * 2 * HALF);
      rb[h] = *reinterpret_cast<const uint2*>(at + (head0 + h) * 2 * HALF + HALF);
    }
  }
  if (here) {
    cs[0] = table[0];
    cs[1] = table[1];
  }
  const float c[4] = {cs[0].x, cs[0].z, cs[1].x, cs[1].z}, sn[4] = {cs[0].y, cs[0].w, cs[1].y, cs[1].w};
#pragma unroll
  for (int h = 0; h < kRopeHeads; ++h) {
    const float2 a0 = unpack_f16x2(ra[h].x), a1 = unpack_f16x2(ra[h].y), b0 = unpack_f16x2(rb[h].x), b1 = unpack_f16x2(rb[h].y);
    float a[4] = {a0.x, a0.y, a1.x, a1.y}, b[4] = {b0.x, b0.y, b1.x, b1.y};
    if (rope.qk_gain) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
#pragma unroll
      for (int o = kLanes / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float r = rsqrtf(ss / (2.0f * HALF) + rope.eps);
      const float* gain = rope.qk_gain + ((head0 + h) * 2 * HALF < rope.q_cols ? 0 : 2 * HALF) + lane * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] *= r * gain[j];
        b[j] *= r * gain[HALF + j];
      }
    }
    if (here && head0 + h < heads) {
      float x[4], y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = a[j] * c[j] - b[j] * sn[j];
        y[j] = b[j] * c[j] + a[j] * sn[j];
      }
      *reinterpret_cast<uint2*>(at + (head0 + h) * 2 * HALF) = make_uint2(pack_f16x2(x[0], x[1]), pack_f16x2(x[2], x[3]));
      *reinterpret_cast<uint2*>(at + (head0 + h) * 2 * HALF + HALF) = make_uint2(pack_f16x2(y[0], y[1]), pack_f16x2(y[2], y[3]));
    }
  }
}

template <int TYPE, int DELTA, bool NORM>
cudaError_t launch_rows(const QuantRows& p, cudaStream_t s) {
  // Pieces a thread. What a thread does once for a row costs as much as ten values, so many rows take four pieces where that leaves
  // four warps to a row (8191 x 3584 bf16 with its norm: 36.1 us, two pieces 39.5; 5377 x 8960 bf16: 28.7, two 38.8, eight, which
  // leave an SM too few rows, 37.9; 1163 x 1536 fp16: two 3.1, four 3.7), fp32 rows two, whose registers are twice as many (2048 x
  // 3584: 8.1 either way; norm of 5377 x 1536: 17.5, four 18.4). Few rows are bound by latency: two pieces, the norm, whose loads are
  // three, one (16 x 1536: 2.0 us against 2.3 with two and 2.8 with four).
  const int units = p.d >> 3;
  const bool few = p.rows <= kNumSMs;
  int nv = units > (TYPE == kF32 ? 2048 : 256) && !few ? 4 : 2;
  if (NORM && few && units <= 1024) nv = 1;
  if (units > 2048) nv = 4;
  const int threads = std::min(nv == 4 ? 640 : 1024, (units + 32 * nv - 1) / (32 * nv) * 32), together = threads == 32 ? 8 : 1;
  const auto kernel = nv == 4   ? quantize_i8_kernel<TYPE, DELTA, NORM, 4>
                      : nv == 2 ? quantize_i8_kernel<TYPE, DELTA, NORM, 2>
                                : quantize_i8_kernel<TYPE, DELTA, NORM, NORM ? 1 : 2>;
  const cudaError_t e = launch_pdl(kernel, dim3(static_cast<unsigned>((static_cast<int64_t>(p.rows) + together - 1) / together)), dim3(threads, together), 0, s, p);
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
  const int units = d >> 4, across = std::min(256, (units + 31) / 32 * 32), down = 256 / across;
  const int64_t blocks = (static_cast<int64_t>(rows) + down - 1) / down;
  const auto kernel = type == kF16 ? dequantize_i8_kernel<kF16> : type == kBF16 ? dequantize_i8_kernel<kBF16> : dequantize_i8_kernel<kF32>;
  const cudaError_t e = launch_pdl(kernel, dim3(static_cast<unsigned>(blocks), std::min(64, (units + across - 1) / across)), dim3(across, down), 0,
                                   s, codes, scales, out, out_stride, rows, d);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_rope_rows(uint16_t* rows, int row_elems, int T, const RopeEpilogue& rope, cudaStream_t s) {
  if (T <= 0) return cudaSuccess;
  if (!rope.table || (rope.half != 32 && rope.half != 64)) return cudaErrorInvalidValue;
  const int groups = (rope.n_rot_cols / (2 * rope.half) + kRopeHeads - 1) / kRopeHeads;
  const int64_t threads = static_cast<int64_t>(T) * groups * (rope.half / 4);
  const cudaError_t e = launch_pdl(rope.half == 64 ? rope_rows_kernel<64> : rope_rows_kernel<32>, dim3(static_cast<unsigned>((threads + 255) / 256)),
                                   dim3(256), 0, s, reinterpret_cast<__half*>(rows), row_elems, T, rope);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace cs
