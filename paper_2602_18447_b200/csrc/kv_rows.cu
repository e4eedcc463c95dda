// Rows of K and V into the pages of a cache, with the rotary turn on the way, and out of them again, for every cache format:
// 16-bit cells, the two 8-bit float formats, and 4-bit codes with a scale and an offset per 64 channels.
// All of it moves bytes: a row is read once and written once, and the arithmetic (a turn, a minimum and a maximum over 64
// channels, a division per channel in the rare case that the product with the reciprocal cannot decide) hides behind it.
#include <cuda_fp8.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "kv4.cuh"

namespace cs {

namespace {

constexpr int kPage = 16;
constexpr float kF16Max = 65504.f;

// Eight consecutive 16-bit values as fp32 (exact).
template <bool BF16>
__device__ __forceinline__ void widen8(const uint4& r, float (&x)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (BF16) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    } else {
      const float2 f = unpack_f16x2(w[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
template <bool BF16>
__device__ __forceinline__ uint4 narrow8(const float (&x)[8]) {
  if (BF16) return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  return make_uint4(pack_f16x2(x[0], x[1]), pack_f16x2(x[2], x[3]), pack_f16x2(x[4], x[5]), pack_f16x2(x[6], x[7]));
}

// What a cache may hold: NaN becomes 0 and magnitudes saturate, because a slot behind a sequence's end is multiplied by a
// zero probability, not skipped.
__device__ __forceinline__ float storable(float v, float most) { return v != v ? 0.f : fminf(fmaxf(v, -most), most); }

// The turn of eight channels `a` of a head's first half against the eight channels `b` half a head further on. Products and sums
// are rounded one by one (no fused multiply-add): the codes that follow sit next to rounding borders, and a plain evaluation of the
// formula has to land on the same side.
__device__ __forceinline__ void turn8(float (&a)[8], float (&b)[8], const float2 (&cs)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = a[i], y = b[i];
    a[i] = __fsub_rn(__fmul_rn(x, cs[i].x), __fmul_rn(y, cs[i].y));
    b[i] = __fadd_rn(__fmul_rn(y, cs[i].x), __fmul_rn(x, cs[i].y));
  }
}

// Minimum and maximum that pass a NaN on.
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float min8(const float (&v)[8]) {
  return min_nan(min_nan(min_nan(v[0], v[1]), min_nan(v[2], v[3])), min_nan(min_nan(v[4], v[5]), min_nan(v[6], v[7])));
}
__device__ __forceinline__ float max8(const float (&v)[8]) {
  return max_nan(max_nan(max_nan(v[0], v[1]), max_nan(v[2], v[3])), max_nan(max_nan(v[4], v[5]), max_nan(v[6], v[7])));
}
// Smallest and largest over the LANES neighbouring lanes of a group; NaN where one is.
template <int LANES>
__device__ __forceinline__ void range_lanes(float& lo, float& hi) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
}

// fp32 values that are whole numbers near 1.5 x 2^23 carry the number in their low bits, and adding rounds to the nearest,
// ties to even.
constexpr float kRound = 12582912.f;
constexpr uint32_t kRoundBits = 0x4B400000u;

// A group's scale and offset from its smallest and largest value. The smallest value is the offset, a fifteenth of the range the
// scale, both rounded to fp16 (half a step of 2^-10 relative; the codes are taken against the rounded pair, so the error stays half
// a code step plus 15 x 2^-11 of one at the far end of the range). The fifteenth is the product with the rounded reciprocal, which is
// what the format says and what caches that were written before hold: a division differs in one group of some 2000, by one fp16 step.
__device__ __forceinline__ void group_params(float lo, float hi, __half& scale, __half& offset) {
  offset = __float2half_rn(lo);
  scale = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f), kKv4MaxScale));
}
// The codes of eight channels. code[i]: kRoundBits + the code.
__device__ __forceinline__ void codes8(const float (&v)[8], __half scale, __half offset, uint32_t (&code)[8]) {
  const float s = __half2float(scale), o = __half2float(offset);
  const float inv15 = s > 0.f ? __fdividef(1.f / 15.f, s) : 0.f;
  float r[8], worst = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float u = __saturatef(__fmul_rn(__fsub_rn(v[i], o), inv15));       // the share of the range, 0 .. 1: clamped for nothing
    r[i] = __fmaf_rn(u, 15.f, kRound);
    worst = fmaxf(worst, fabsf(__fmaf_rn(u, 15.f, -__fsub_rn(r[i], kRound))));
  }
  // The reciprocal's 2^-22 and two roundings of 2^-24 move a quotient of up to 15 by less than 6e-6: only that close to a border does
  // the quotient itself have to decide.
  if (worst > 0.49999f && s > 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      r[i] = fminf(fmaxf(__fadd_rn(__fdiv_rn(__fsub_rn(v[i], o), s), kRound), kRound), kRound + 15.f);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) code[i] = __float_as_uint(r[i]);
}
// The codes of a thread's two chunks (eight channels each, half a head apart) and the parameters of their groups, which for
// HD = 64 are one. NaN, infinities and what the format cannot hold are rare: the whole warp goes round again with storable values.
template <int HD>
__device__ __forceinline__ void quantise(float (&a)[8], float (&b)[8], uint32_t (&ca)[8], uint32_t (&cb)[8], __half (&scale)[2],
                                         __half (&offset)[2]) {
  for (bool again = false;; again = true) {
    float lo0 = min8(a), hi0 = max8(a), lo1 = min8(b), hi1 = max8(b);
    if (HD == 64) {
      lo0 = lo1 = min_nan(lo0, lo1);
      hi0 = hi1 = max_nan(hi0, hi1);
      range_lanes<4>(lo0, hi0);
      lo1 = lo0;
      hi1 = hi0;
    } else {
      range_lanes<8>(lo0, hi0);
      range_lanes<8>(lo1, hi1);
    }
    const bool fits = min_nan(lo0, lo1) >= -kF16Max && max_nan(hi0, hi1) <= kF16Max;
    if (again || !__any_sync(0xffffffffu, !fits)) {
      group_params(lo0, hi0, scale[0], offset[0]);
      group_params(lo1, hi1, scale[1], offset[1]);
      break;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a[i] = storable(a[i], kF16Max);
      b[i] = storable(b[i], kF16Max);
    }
  }
  codes8(a, scale[0], offset[0], ca);
  codes8(b, scale[1], offset[1], cb);
}
// sum of code[i] << at(i) without the bits that kRoundBits adds
template <typename At>
__device__ __forceinline__ uint32_t pack_codes(const uint32_t (&code)[8], At at) {
  uint32_t w = 0, extra = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w += code[i] << at(i);
    extra += kRoundBits << at(i);
  }
  return w - extra;
}

template <int FMT>
__device__ __forceinline__ uint8_t fp8_of(float v) {
  return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, FMT == CS_KV_FMT_E4M3 ? __NV_E4M3 : __NV_E5M2);
}

// Bytes of a page's image in shared memory (full pages are put together there and leave in 16-byte stores).
template <int HD, int FMT>
__host__ __device__ constexpr int image_bytes() {
  return FMT == CS_KV_FMT_INT4 ? Kv4<HD>::kBlock : FMT == CS_KV_FMT_16BIT ? 16 : kPage * HD;
}

// Eight channels of V of one token (chunk c) into a 4-bit block: its tile is c / 2, this thread's chunk is the tile's lower (c even)
// or upper half, and of the eight bytes it writes four. own, other: this chunk's and the neighbouring lane's codes.
template <int HD>
__device__ __forceinline__ void put_v4(uint8_t* dst, int slot, int c, uint32_t own, uint32_t other) {
  using L = Kv4<HD>;
  const uint32_t low = c & 1 ? other >> 16 : own, high = c & 1 ? own >> 16 : other;
  const uint32_t even = (low & 0x0F0Fu) | (high & 0x0F0Fu) << 4, odd = (low >> 4 & 0x0F0Fu) | (high & 0xF0F0u);
  const int g0 = 4 * (c & 1);
  dst[L::kVCodes + L::v_byte(slot, c >> 1, g0)] = static_cast<uint8_t>(even);
  dst[L::kVCodes + L::v_byte(slot, c >> 1, g0 + 1)] = static_cast<uint8_t>(odd);
  dst[L::kVCodes + L::v_byte(slot, c >> 1, g0 + 2)] = static_cast<uint8_t>(even >> 8);
  dst[L::kVCodes + L::v_byte(slot, c >> 1, g0 + 3)] = static_cast<uint8_t>(odd >> 8);
}

// One CTA: the tokens of one block (consecutive positions of one page). A thread has two chunks of eight channels half a head apart,
// which turn against each other, of one token, and loops over the CTA's share of the heads with the token's cosines and sines in
// registers and the next head's rows on their way. blockIdx.y < kv_parts: K and V heads; behind them, query heads.
// Bound by memory and instructions alike: 4-bit rows of 22.9 K tokens x 8 heads with 16 query heads (0.32 GB in and out) take
// 69 us, 0.71 of the copy bandwidth; 16-bit ones of 2 heads with 12 query heads (0.2 GB) 34.7 us, 0.88. What counted: two chunks a
// thread (no exchange between lanes for the turn), rounding by addition with one border check for eight channels (a rounding, range
// check and branch per channel: 140 us), whole pages through shared memory.
template <int HD, int FMT, bool BF16>
__global__ void __launch_bounds__(HD, 640 / HD) kv_append_kernel(const KvAppendParams p) {
  constexpr int CH = HD / 8, HALF = CH / 2;          // chunks of a row; threads of a token
  constexpr int kImage = image_bytes<HD, FMT>();
  __shared__ __align__(16) uint8_t images[2 * kImage];
  pdl_launch_dependents();
  const KvBlock blk = p.blocks[blockIdx.x];
  const int i = threadIdx.x / HALF, c = threadIdx.x % HALF;
  const bool active = i < blk.n;
  const int64_t tok = blk.tok0 + i;
  float2 cs[8];
  const bool turn = p.rope != nullptr;
  pdl_wait();
  if (turn && active) {
    const float4* r = reinterpret_cast<const float4*>(p.rope + tok * (HD / 2) + c * 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 f = r[j];
      cs[2 * j] = make_float2(f.x, f.y);
      cs[2 * j + 1] = make_float2(f.z, f.w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[j] = make_float2(1.f, 0.f);
  }
  const uint4 zero = make_uint4(0, 0, 0, 0);
  auto load = [&](const uint16_t* src, bool there, uint4 (&r)[2]) {
    r[0] = there ? *reinterpret_cast<const uint4*>(src) : zero;
    r[1] = there ? *reinterpret_cast<const uint4*>(src + HD / 2) : zero;
  };
  if (static_cast<int>(blockIdx.y) >= p.kv_parts) {
    const int part = blockIdx.y - p.kv_parts;
    const int h0 = part * p.q_heads_per_part, h1 = min(p.n_q_heads, h0 + p.q_heads_per_part);
    const uint16_t* src = p.q + tok * p.q_stride + c * 8;
    uint16_t* dst = p.q_out + tok * p.q_out_stride + c * 8;
    // two heads a round, the next two requested before these are stored (q_out may be q: a thread writes what it alone reads)
    uint4 raw[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j) load(src + (h0 + j) * HD, active && h0 + j < h1, raw[j]);
    for (int h = h0; h < h1; h += 2) {
      uint4 next[2][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) load(src + (h + 2 + j) * HD, active && h + 2 + j < h1, next[j]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float x[8], y[8];
        widen8<BF16>(raw[j][0], x);
        widen8<BF16>(raw[j][1], y);
        turn8(x, y, cs);
        if (active && h + j < h1) {
          *reinterpret_cast<uint4*>(dst + (h + j) * HD) = narrow8<BF16>(x);
          *reinterpret_cast<uint4*>(dst + (h + j) * HD + HD / 2) = narrow8<BF16>(y);
        }
        raw[j][0] = next[j][0];
        raw[j][1] = next[j][1];
      }
    }
    return;
  }
  const int slot = (blk.pos0 + i) % kPage;
  const int page = p.table[static_cast<size_t>(blk.seq) * p.max_pages_per_seq + blk.pos0 / kPage];
  const bool ok = debug_in_range(page >= 0 && page < p.num_pages && blk.pos0 / kPage < p.max_pages_per_seq, p.status);
  const bool whole = blk.n == kPage && FMT != CS_KV_FMT_16BIT;
  const int h0 = blockIdx.y * p.kv_heads_per_part, h1 = min(p.n_kv_heads, h0 + p.kv_heads_per_part);
  const uint16_t* src_k = p.k + tok * p.k_stride + c * 8;
  const uint16_t* src_v = p.v + tok * p.v_stride + c * 8;
  uint4 rk[2], rv[2];
  load(src_k + h0 * HD, active, rk);
  load(src_v + h0 * HD, active, rv);
  uint8_t* image = images;
  for (int h = h0; h < h1; ++h) {
    uint4 next_k[2], next_v[2];
    load(src_k + (h + 1) * HD, active && h + 1 < h1, next_k);
    load(src_v + (h + 1) * HD, active && h + 1 < h1, next_v);
    float a[8], b[8];
    widen8<BF16>(rk[0], a);
    widen8<BF16>(rk[1], b);
    if (turn) turn8(a, b, cs);
    const size_t ph = static_cast<size_t>(page) * p.n_kv_heads + h;
    if (FMT == CS_KV_FMT_16BIT) {
      // the 16-bit cache holds bf16 values in the fp16 encoding
      auto put = [&](uint8_t* pool) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          a[j] = storable(__bfloat162float(__float2bfloat16_rn(a[j])), kF16Max);
          b[j] = storable(__bfloat162float(__float2bfloat16_rn(b[j])), kF16Max);
        }
        uint16_t* dst = reinterpret_cast<uint16_t*>(pool) + (ph * kPage + slot) * HD + c * 8;
        if (active && ok) {
          *reinterpret_cast<uint4*>(dst) = narrow8<false>(a);
          *reinterpret_cast<uint4*>(dst + HD / 2) = narrow8<false>(b);
        }
      };
      put(p.pool_k);
      widen8<BF16>(rv[0], a);
      widen8<BF16>(rv[1], b);
      put(p.pool_v);
    } else if (FMT == CS_KV_FMT_INT4) {
      using L = Kv4<HD>;
      uint8_t* block = p.pool_k + ph * L::kBlock;
      __half ks[2], ko[2], vs[2], vo[2];
      uint32_t ca[8], cb[8];
      quantise<HD>(a, b, ca, cb, ks, ko);
      // kv4.cuh: neighbouring channels side by side in the two halves of the word
      const uint32_t kw0 = pack_codes(ca, [](int j) { return 4 * (j / 2) + 16 * (j & 1); });
      const uint32_t kw1 = pack_codes(cb, [](int j) { return 4 * (j / 2) + 16 * (j & 1); });
      widen8<BF16>(rv[0], a);
      widen8<BF16>(rv[1], b);
      quantise<HD>(a, b, ca, cb, vs, vo);
      const uint32_t vc0 = pack_codes(ca, [](int j) { return 4 * j; }), vc1 = pack_codes(cb, [](int j) { return 4 * j; });
      const uint32_t vp0 = __shfl_xor_sync(0xffffffffu, vc0, 1), vp1 = __shfl_xor_sync(0xffffffffu, vc1, 1);
      auto put = [&](uint8_t* dst) {
        *reinterpret_cast<uint32_t*>(dst + L::k_word(slot, c * 8)) = kw0;
        *reinterpret_cast<uint32_t*>(dst + L::k_word(slot, HD / 2 + c * 8)) = kw1;
        put_v4<HD>(dst, slot, c, vc0, vp0);
        put_v4<HD>(dst, slot, HALF + c, vc1, vp1);
        if (c < L::kGroups) {                        // thread 0 writes the first group's parameters, thread 1 the second's
          *reinterpret_cast<__half*>(dst + L::kKScale + L::k_param(slot, c)) = c ? ks[1] : ks[0];
          *reinterpret_cast<__half*>(dst + L::kKOffset + L::k_param(slot, c)) = c ? ko[1] : ko[0];
          *reinterpret_cast<__half*>(dst + L::v_scale(slot, c)) = c ? vs[1] : vs[0];
          *reinterpret_cast<__half*>(dst + L::v_offset(slot, c)) = c ? vo[1] : vo[0];
        }
      };
      if (whole) {
        put(image);
        __syncthreads();
        if (ok)
          for (int j = threadIdx.x; j < L::kBlock / 16; j += HD)
            reinterpret_cast<uint4*>(block)[j] = reinterpret_cast<const uint4*>(image)[j];
      } else if (active && ok) {
        put(block);
      }
    } else {
      constexpr float most = FMT == CS_KV_FMT_E4M3 ? 448.f : 57344.f;
      uint8_t* kt = p.pool_k + (ph * kPage + slot) * HD + c * 8;
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j >> 2] |= static_cast<uint32_t>(fp8_of<FMT>(storable(a[j], most))) << (8 * (j & 3));
        w[2 + (j >> 2)] |= static_cast<uint32_t>(fp8_of<FMT>(storable(b[j], most))) << (8 * (j & 3));
      }
      if (active && ok) {
        *reinterpret_cast<uint2*>(kt) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(kt + HD / 2) = make_uint2(w[2], w[3]);
      }
      widen8<BF16>(rv[0], a);
      widen8<BF16>(rv[1], b);
      uint8_t* vt = p.pool_v + ph * kPage * HD;                  // V pages are kept transposed, [HD][16]
      auto put = [&](uint8_t* dst) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dst[(c * 8 + j) * kPage + slot] = fp8_of<FMT>(storable(a[j], most));
          dst[(HD / 2 + c * 8 + j) * kPage + slot] = fp8_of<FMT>(storable(b[j], most));
        }
      };
      if (whole) {
        put(image);
        __syncthreads();
        if (ok) reinterpret_cast<uint4*>(vt)[threadIdx.x] = reinterpret_cast<const uint4*>(image)[threadIdx.x];
      } else if (active && ok) {
        put(vt);
      }
    }
    image = image == images ? images + kImage : images;   // the other one was read before the barrier just passed
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      rk[j] = next_k[j];
      rv[j] = next_v[j];
    }
  }
}

template <int FMT>
__device__ __forceinline__ float fp8_value(uint8_t b) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw(b, FMT == CS_KV_FMT_E4M3 ? __NV_E4M3 : __NV_E5M2);
  return __half2float(__half(h));
}

// Two codes as exact fp16 numbers -> the values that they stand for: fp16 in one fused rounding, bf16 through fp32. A code of 15 may
// stand for up to 65524 (the offset of a turned row rounds up by 16, 15 scales by 4): fp16 holds it at 65504, not as an infinity.
template <bool BF16>
__device__ __forceinline__ uint32_t value2(uint32_t c, uint32_t scale2, uint32_t offset2) {
  if (BF16) {
    const float2 f = unpack_f16x2(c), s = unpack_f16x2(scale2), o = unpack_f16x2(offset2);
    return pack_bf16x2(fmaf(f.x, s.x, o.x), fmaf(f.y, s.y, o.y));
  }
  const uint32_t most = 0x7BFF7BFFu;
  const __half2 r = __hmin2(__hfma2(*reinterpret_cast<const __half2*>(&c), *reinterpret_cast<const __half2*>(&scale2),
                                    *reinterpret_cast<const __half2*>(&offset2)), *reinterpret_cast<const __half2*>(&most));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Nibbles 0 and 4 (1024 + c), or 1 and 5 (64 + c), of w as exact fp16 numbers.
__device__ __forceinline__ uint32_t nibbles(uint32_t w, bool high) {
  uint32_t r;
  if (high) asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(0x00F000F0u), "r"(0x54005400u));
  else asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(0x000F000Fu), "r"(0x64006400u));
  const uint32_t base = high ? 0xD400D400u : 0xE400E400u;
  const __half2 c = __hadd2(*reinterpret_cast<const __half2*>(&r), *reinterpret_cast<const __half2*>(&base));
  return *reinterpret_cast<const uint32_t*>(&c);
}
__device__ __forceinline__ uint32_t splat(uint32_t halves, int which) {
  return __byte_perm(halves, halves, which ? 0x3232 : 0x1010);
}

// One warp: rows of a 4-bit block as values. row(slot) says where a slot's row goes: the element offset of K and V, or negative
// for a slot that is not wanted. The words are the attention's, so that a mask takes two channels (K) or two words give two
// channels of four keys (V).
template <int HD, bool BF16, typename Row>
__device__ __forceinline__ void block_rows(const uint8_t* b, int lane, uint16_t* out_k, uint16_t* out_v, Row row) {
  using L = Kv4<HD>;
  constexpr int CH = HD / 8, kRows = 32 / CH, kRounds = kPage / kRows;       // K: rows of 8-channel chunks that a warp has at once
  constexpr int MT = HD / 16;
  const int c = lane % CH, q = lane / MT & 3, mt = lane % MT;
  // every load first: unwanted slots cost a few bytes, a load behind a branch costs its latency
  uint32_t kw[kRounds], w[8];
  uint16_t ks[kRounds], ko[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int slot = r * kRows + lane / CH;
    kw[r] = *reinterpret_cast<const uint32_t*>(b + L::k_word(slot, c * 8));
    ks[r] = *reinterpret_cast<const uint16_t*>(b + L::kKScale + L::k_param(slot, c / 8));
    ko[r] = *reinterpret_cast<const uint16_t*>(b + L::kKOffset + L::k_param(slot, c / 8));
  }
  // V: lane (q, mt) has the 16 channels of tile mt of keys 2 q, 2 q + 8, 2 q + 1, 2 q + 9 (HD = 64: half the lanes)
#pragma unroll
  for (int g = 0; g < 8; ++g)
    w[g] = *reinterpret_cast<const uint32_t*>(b + L::kVCodes + (mt / 4) * 512 + L::v_chunk(g, q) * 16 + (mt % 4) * 4);
  const uint2 s4 = *reinterpret_cast<const uint2*>(b + L::v_scale(2 * q, mt / 4));
  const uint2 o4 = *reinterpret_cast<const uint2*>(b + L::v_offset(2 * q, mt / 4));
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t at = row(r * kRows + lane / CH);
    const uint32_t s = splat(ks[r], 0), o = splat(ko[r], 0), w8 = kw[r] >> 8;
    if (at >= 0)
      *reinterpret_cast<uint4*>(out_k + at + c * 8) =
          make_uint4(value2<BF16>(nibbles(kw[r], false), s, o), value2<BF16>(nibbles(kw[r], true), s, o),
                     value2<BF16>(nibbles(w8, false), s, o), value2<BF16>(nibbles(w8, true), s, o));
  }
  if (lane / MT >= 4) return;
#pragma unroll
  for (int byte = 0; byte < 4; ++byte) {
    const int odd = byte >> 1, up = byte & 1;
    const int64_t at = row(2 * q + odd + 8 * up);
    if (at < 0) continue;
    const uint32_t s = splat(up ? s4.y : s4.x, odd), o = splat(up ? o4.y : o4.x, odd);
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t x = __byte_perm(w[2 * j], w[2 * j + 1], byte * 0x0011 + (4 + byte) * 0x1100);
      lo[j] = value2<BF16>(nibbles(x, false), s, o);
      hi[j] = value2<BF16>(nibbles(x, true), s, o);
    }
    *reinterpret_cast<uint4*>(out_v + at + mt * 16) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    *reinterpret_cast<uint4*>(out_v + at + mt * 16 + 8) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  }
}

// Page id of a listed place, or -1 outside the sequence's pages.
__device__ __forceinline__ int listed_page(const KvReadParams& p, int row, int& pos) {
  const int seq = p.tok_seq[row];
  pos = p.tok_pos[row];
  if (seq < 0 || seq >= p.max_seqs || pos < 0 || pos / kPage >= p.max_pages_per_seq) return -1;
  const int n = __ldg(p.n_pages + seq);      // beside the next load, not behind it
  const int page = __ldg(p.table + static_cast<size_t>(seq) * p.max_pages_per_seq + pos / kPage);
  return (page < p.num_pages) & (pos / kPage < n) ? page : -1;
}

// Rows listed by (sequence, position) out of a 16-bit or 8-bit cache: one thread per row and 8 channels. A place outside the sequence's
// pages gives a row of zeros and raises the range bit of the status word.
template <int HD, int FMT, bool BF16>
__global__ void __launch_bounds__(2 * HD) kv_read_kernel(const KvReadParams p) {
  constexpr int CH = HD / 8;
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x * kPage + threadIdx.x / CH, c = threadIdx.x % CH, h = blockIdx.y;
  if (row >= p.T) return;
  int pos;
  const int page = listed_page(p, row, pos);
  if (page < 0 && c == 0 && h == 0) atomicOr(p.status, kStatusRange);
  const int slot = pos & (kPage - 1);
  float k[8] = {}, v[8] = {};
  if (page >= 0) {
    const size_t ph = static_cast<size_t>(page) * p.n_kv_heads + h;
    if (FMT == CS_KV_FMT_16BIT) {
      const size_t at = (ph * kPage + slot) * HD + c * 8;
      widen8<false>(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.pool_k) + at), k);
      widen8<false>(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.pool_v) + at), v);
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(p.pool_k + (ph * kPage + slot) * HD + c * 8);
      const uint8_t* vt = p.pool_v + ph * kPage * HD;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        k[j] = fp8_value<FMT>(static_cast<uint8_t>((j < 4 ? w.x : w.y) >> (8 * (j & 3))));
        v[j] = fp8_value<FMT>(vt[(c * 8 + j) * kPage + slot]);
      }
    }
  }
  const size_t at = (static_cast<size_t>(row) * p.n_kv_heads + h) * HD + c * 8;
  *reinterpret_cast<uint4*>(p.out_k + at) = narrow8<BF16>(k);
  *reinterpret_cast<uint4*>(p.out_v + at) = narrow8<BF16>(v);
}

// The same out of a 4-bit cache. ROWS listed rows a CTA: runs of rows that climb through one page are found first, then a warp takes a
// run and reads its block's words once for all of them (a V code by itself is half a byte; row by row took 44 us for 22.9 K
// rows x 8 heads, by runs 26 us, 0.72 of the copy bandwidth).
template <int HD, bool BF16, int ROWS, int THREADS>
__global__ void __launch_bounds__(THREADS) kv_read4_kernel(const KvReadParams p) {
  static_assert(ROWS <= 64 && THREADS >= ROWS, "one thread per row, two ballots");
  __shared__ int16_t run_row[ROWS][kPage];      // by run and slot: row of the CTA, or -1
  __shared__ int run_page[ROWS];
  __shared__ int ends[ROWS], n_first;
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31;
  for (int j = tid; j < ROWS * kPage / 2; j += THREADS) reinterpret_cast<int*>(run_row)[j] = -1;
  pdl_wait();
  const int row0 = blockIdx.x * ROWS, n = min(ROWS, p.T - row0);
  int page = -1, pos = 0, key = -1;
  if (tid < n) {
    page = listed_page(p, row0 + tid, pos);
    if (page < 0 && blockIdx.y == 0) atomicOr(p.status, kStatusRange);
    key = page < 0 ? -1 : page * kPage + (pos & (kPage - 1));     // num_pages x heads x 16 is below 2^31
  }
  if (tid < ROWS) ends[tid] = key;
  __syncthreads();
  // a run begins where the page changes or the slot does not climb; a place outside the table is a run of its own
  bool begins = false;
  if (tid < n) {
    const int before = tid > 0 ? ends[tid - 1] : -1;
    begins = key < 0 || before < 0 || before / kPage != page || before >= key;
  }
  const uint32_t bits = __ballot_sync(0xffffffffu, begins);
  if (tid == 31) n_first = __popc(bits);          // at most 64 rows: two warps
  __syncthreads();
  const int run = __popc(bits & (0xffffffffu >> (31 - lane))) - 1 + (tid >= 32 ? n_first : 0);
  if (tid < n) {
    if (begins) run_page[run] = page;
    run_row[run][page < 0 ? 0 : key & (kPage - 1)] = static_cast<int16_t>(tid);
  }
  if (tid == n - 1) ends[0] = run + 1;
  __syncthreads();
  const int runs = ends[0], h = blockIdx.y;
  const int64_t stride = static_cast<int64_t>(p.n_kv_heads) * HD;
  for (int r = tid >> 5; r < runs; r += THREADS / 32) {
    const int64_t base = static_cast<int64_t>(row0) * stride + h * HD;
    const int pg = run_page[r];
    if (pg < 0) {
      const int64_t at = base + run_row[r][0] * stride;
      for (int c = lane; c < HD / 8; c += 32) {
        *reinterpret_cast<uint4*>(p.out_k + at + c * 8) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(p.out_v + at + c * 8) = make_uint4(0, 0, 0, 0);
      }
      continue;
    }
    block_rows<HD, BF16>(p.pool_k + (static_cast<size_t>(pg) * p.n_kv_heads + h) * Kv4<HD>::kBlock, lane, p.out_k, p.out_v,
                         [&](int slot) -> int64_t { return run_row[r][slot] < 0 ? -1 : base + run_row[r][slot] * stride; });
  }
}

// Whole pages of the 4-bit cache as fp16 pages of a scratch pool (the layout of the 16-bit cache), in the order of the list: what
// the tensor-core attention of long steps reads. One warp per (listed page, kv head).
template <int HD>
__global__ void __launch_bounds__(128) kv_expand_kernel(const uint8_t* pool, const int32_t* __restrict__ pages,
                                                       int n_pages, uint16_t* out_k, uint16_t* out_v,
                                                       int n_kv_heads, int num_pages, uint32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t task = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (task >= static_cast<int64_t>(n_pages) * n_kv_heads) return;
  const int page = __ldg(pages + task / n_kv_heads), h = static_cast<int>(task % n_kv_heads);
  if (!debug_in_range(page >= 0 && page < num_pages, status)) return;
  block_rows<HD, false>(pool + (static_cast<size_t>(page) * n_kv_heads + h) * Kv4<HD>::kBlock, threadIdx.x & 31, out_k, out_v,
                        [&](int slot) -> int64_t { return (task * kPage + slot) * HD; });
}

// The new tokens' keys and values out of the 4-bit cache into the K and V columns of a fused fp16 matrix. One warp per (block of
// tokens of one page, kv head).
template <int HD>
__global__ void __launch_bounds__(128) kv_blocks_kernel(const uint8_t* pool, const KvBlock* __restrict__ blocks,
                                                       int n_blocks, const int32_t* __restrict__ table, int max_pages_per_seq,
                                                       uint16_t* out_k, uint16_t* out_v, int64_t stride,
                                                       int n_kv_heads, int num_pages, uint32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t task = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (task >= static_cast<int64_t>(n_blocks) * n_kv_heads) return;
  const KvBlock blk = blocks[task / n_kv_heads];
  const int h = static_cast<int>(task % n_kv_heads), slot0 = blk.pos0 % kPage;
  const int page = __ldg(table + static_cast<size_t>(blk.seq) * max_pages_per_seq + blk.pos0 / kPage);
  if (!debug_in_range(page >= 0 && page < num_pages && blk.pos0 / kPage < max_pages_per_seq, status)) return;
  block_rows<HD, false>(pool + (static_cast<size_t>(page) * n_kv_heads + h) * Kv4<HD>::kBlock, threadIdx.x & 31, out_k, out_v,
                        [&](int slot) -> int64_t {
                          const int i = slot - slot0;
                          return i >= 0 && i < blk.n ? (blk.tok0 + i) * stride + h * HD : -1;
                        });
}

// Up to three row sources side by side into one matrix, in 16-byte pieces, fp16 or bf16 on either side (bf16 -> fp16 is exact for
// magnitudes in [2^-14, 65504]). Sources behind the first are keys and values: non-finite ones are held as the cache holds them.
template <bool FROM_BF16, bool TO_BF16>
__global__ void rows_copy_kernel(const RowsCopy p, int64_t total) {
  pdl_launch_dependents();
  pdl_wait();
  const int pieces = p.cols[0] + p.cols[1] + p.cols[2];
  for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < total;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t row = i / pieces;
    const int c = static_cast<int>(i - row * pieces);
    const int which = c < p.cols[0] ? 0 : c < p.cols[0] + p.cols[1] ? 1 : 2;
    const int at = c - (which > 0 ? p.cols[0] : 0) - (which > 1 ? p.cols[1] : 0);
    float x[8];
    widen8<FROM_BF16>(*reinterpret_cast<const uint4*>(p.src[which] + row * p.stride[which] + at * 8), x);
    if (which > 0)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = storable(x[j], kF16Max);
    *reinterpret_cast<uint4*>(p.dst + row * p.dst_stride + c * 8) = narrow8<TO_BF16>(x);
  }
}

template <int HD, int FMT>
cudaError_t append_fmt(const KvAppendParams& p, dim3 grid, cudaStream_t s) {
  return p.src_bf16 ? launch_pdl(kv_append_kernel<HD, FMT, true>, grid, dim3(HD), 0, s, p)
                    : launch_pdl(kv_append_kernel<HD, FMT, false>, grid, dim3(HD), 0, s, p);
}
template <int HD>
cudaError_t append_hd(const KvAppendParams& p, int format, dim3 grid, cudaStream_t s) {
  switch (format) {
    case CS_KV_FMT_16BIT: return append_fmt<HD, CS_KV_FMT_16BIT>(p, grid, s);
    case CS_KV_FMT_E4M3: return append_fmt<HD, CS_KV_FMT_E4M3>(p, grid, s);
    case CS_KV_FMT_E5M2: return append_fmt<HD, CS_KV_FMT_E5M2>(p, grid, s);
    case CS_KV_FMT_INT4: return append_fmt<HD, CS_KV_FMT_INT4>(p, grid, s);
    default: return cudaErrorInvalidValue;
  }
}

template <int HD, int FMT>
cudaError_t read_fmt(const KvReadParams& p, dim3 grid, cudaStream_t s) {
  return p.dst_bf16 ? launch_pdl(kv_read_kernel<HD, FMT, true>, grid, dim3(2 * HD), 0, s, p)
                    : launch_pdl(kv_read_kernel<HD, FMT, false>, grid, dim3(2 * HD), 0, s, p);
}
template <int HD>
cudaError_t read_hd(const KvReadParams& p, int format, dim3 grid, cudaStream_t s) {
  switch (format) {
    case CS_KV_FMT_16BIT: return read_fmt<HD, CS_KV_FMT_16BIT>(p, grid, s);
    case CS_KV_FMT_E4M3: return read_fmt<HD, CS_KV_FMT_E4M3>(p, grid, s);
    case CS_KV_FMT_E5M2: return read_fmt<HD, CS_KV_FMT_E5M2>(p, grid, s);
    case CS_KV_FMT_INT4: {
      // many rows: 64 a CTA, so that few pages are met by two CTAs; few: 16 rows for eight warps, so that rows of as many pages
      // (one token of each sequence) are not read one after the other
      if (static_cast<int64_t>((p.T + 63) / 64) * p.n_kv_heads >= 2 * kNumSMs) {
        const dim3 grid4((p.T + 63) / 64, p.n_kv_heads);
        return p.dst_bf16 ? launch_pdl(kv_read4_kernel<HD, true, 64, 128>, grid4, dim3(128), 0, s, p)
                          : launch_pdl(kv_read4_kernel<HD, false, 64, 128>, grid4, dim3(128), 0, s, p);
      }
      const dim3 grid4((p.T + 15) / 16, p.n_kv_heads);
      return p.dst_bf16 ? launch_pdl(kv_read4_kernel<HD, true, 16, 256>, grid4, dim3(256), 0, s, p)
                        : launch_pdl(kv_read4_kernel<HD, false, 16, 256>, grid4, dim3(256), 0, s, p);
    }
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace

cudaError_t launch_kv_append(KvAppendParams p, int format, int hd, int n_blocks, cudaStream_t s) {
  if (n_blocks <= 0) return cudaSuccess;
  // few blocks: one head per CTA, for latency; many: several, which read the token's cosines and sines once
  int per = 1;
  while (per < 8 && static_cast<long>(n_blocks) * ((p.n_kv_heads + 2 * per - 1) / (2 * per)) >= 8L * kNumSMs) per *= 2;
  p.kv_heads_per_part = per;
  p.kv_parts = (p.n_kv_heads + per - 1) / per;
  p.q_heads_per_part = 2 * per;
  const int q_parts = p.q ? (p.n_q_heads + 2 * per - 1) / (2 * per) : 0;
  const dim3 grid(n_blocks, p.kv_parts + q_parts);
  const cudaError_t e = hd == 128 ? append_hd<128>(p, format, grid, s) : append_hd<64>(p, format, grid, s);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv_read(const KvReadParams& p, int format, int hd, cudaStream_t s) {
  if (p.T <= 0) return cudaSuccess;
  const int blocks = (p.T + kPage - 1) / kPage;
  const dim3 grid(blocks, p.n_kv_heads);
  const cudaError_t e = hd == 128 ? read_hd<128>(p, format, grid, s) : read_hd<64>(p, format, grid, s);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv_expand(const uint8_t* pool, const int32_t* pages, int n_pages, uint16_t* out_k, uint16_t* out_v,
                             int n_kv_heads, int hd, int num_pages, uint32_t* status, cudaStream_t s) {
  if (n_pages <= 0) return cudaSuccess;
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(n_pages) * n_kv_heads + 3) / 4)), block(128);
  const cudaError_t e =
      hd == 128 ? launch_pdl(kv_expand_kernel<128>, grid, block, 0, s, pool, pages, n_pages, out_k, out_v, n_kv_heads, num_pages, status)
                : launch_pdl(kv_expand_kernel<64>, grid, block, 0, s, pool, pages, n_pages, out_k, out_v, n_kv_heads, num_pages, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv_blocks(const uint8_t* pool, const KvBlock* blocks, int n_blocks, const int32_t* table, int max_pages_per_seq,
                             uint16_t* out_k, uint16_t* out_v, int64_t stride, int n_kv_heads, int hd, int num_pages,
                             uint32_t* status, cudaStream_t s) {
  if (n_blocks <= 0) return cudaSuccess;
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(n_blocks) * n_kv_heads + 3) / 4)), block(128);
  const cudaError_t e = hd == 128 ? launch_pdl(kv_blocks_kernel<128>, grid, block, 0, s, pool, blocks, n_blocks, table,
                                               max_pages_per_seq, out_k, out_v, stride, n_kv_heads, num_pages, status)
                                  : launch_pdl(kv_blocks_kernel<64>, grid, block, 0, s, pool, blocks, n_blocks, table,
                                               max_pages_per_seq, out_k, out_v, stride, n_kv_heads, num_pages, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_rows_copy(const RowsCopy& p, bool from_bf16, bool to_bf16, int rows, cudaStream_t s) {
  const int64_t total = static_cast<int64_t>(rows) * (p.cols[0] + p.cols[1] + p.cols[2]);
  if (total <= 0) return cudaSuccess;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((total + 255) / 256, 8 * kNumSMs))), block(256);
  cudaError_t e;
  if (from_bf16) e = to_bf16 ? launch_pdl(rows_copy_kernel<true, true>, grid, block, 0, s, p, total)
                             : launch_pdl(rows_copy_kernel<true, false>, grid, block, 0, s, p, total);
  else e = to_bf16 ? launch_pdl(rows_copy_kernel<false, true>, grid, block, 0, s, p, total)
                   : launch_pdl(rows_copy_kernel<false, false>, grid, block, 0, s, p, total);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace cs
