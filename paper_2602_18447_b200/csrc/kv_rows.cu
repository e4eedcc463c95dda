// Rows of K and V into the pages of a cache, with the rotary turn on the way, and out of them again, for every cache format:
// 16-bit cells, the two 8-bit float formats, and 4-bit codes with a scale and an offset per 64 channels.
// All of it moves bytes: a row is read once and written once, and the arithmetic (a turn, a minimum and a maximum over 64
// channels, a division per channel in the rare case that the product with the reciprocal cannot decide) hides behind it.
#include <cuda_fp8.h>

#include "common.cuh"
#include "kernels.h"
#include "kv4.cuh"

namespace cs {

namespace {

constexpr int kPage = 16;
constexpr float kF16Max = 65504.f;

// Eight consecutive 16-bit values as fp32 (exact).
__device__ __forceinline__ void widen8(const uint4& r, bool bf16, float (&x)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (bf16) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    } else {
      const float2 f = unpack_f16x2(w[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
__device__ __forceinline__ uint4 narrow8(const float (&x)[8], bool bf16) {
  if (bf16) return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  return make_uint4(pack_f16x2(x[0], x[1]), pack_f16x2(x[2], x[3]), pack_f16x2(x[4], x[5]), pack_f16x2(x[6], x[7]));
}

// What a cache may hold: NaN becomes 0 and magnitudes saturate, because a slot behind a sequence's end is multiplied by a
// zero probability, not skipped.
__device__ __forceinline__ float storable(float v, float most) { return v != v ? 0.f : fminf(fmaxf(v, -most), most); }

// The turn of eight channels: `x` holds this thread's channels, the partner thread (lane ^ DIST) the channels half a head
// away. Products and sums are rounded one by one (no fused multiply-add): the codes that follow sit next to rounding borders,
// and a plain evaluation of the formula has to land on the same side.
template <int HD>
__device__ __forceinline__ void turn8(float (&x)[8], const uint4& raw, bool bf16, const float2 (&cs)[8], bool first_half) {
  constexpr int DIST = HD / 16;
  uint4 other;
  other.x = __shfl_xor_sync(0xffffffffu, raw.x, DIST);
  other.y = __shfl_xor_sync(0xffffffffu, raw.y, DIST);
  other.z = __shfl_xor_sync(0xffffffffu, raw.z, DIST);
  other.w = __shfl_xor_sync(0xffffffffu, raw.w, DIST);
  float y[8];
  widen8(other, bf16, y);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = __fmul_rn(y[i], cs[i].y);
    x[i] = first_half ? __fsub_rn(__fmul_rn(x[i], cs[i].x), t) : __fadd_rn(__fmul_rn(x[i], cs[i].x), t);
  }
}

// Codes of eight channels, 4 bits each (channel i in nibble i), and the scale and offset of their group of 64 channels,
// which eight neighbouring lanes hold. The smallest value is the offset, a fifteenth of the range the scale, both rounded to
// fp16 (half a step of 2^-10 relative; the codes are taken against the rounded pair, so the error stays half a code step
// plus 15 x 2^-11 of one at the far end of the range).
__device__ __forceinline__ uint32_t quantise8(const float (&v)[8], __half& scale, __half& offset) {
  float lo = v[0], hi = v[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, v[i]);
    hi = fmaxf(hi, v[i]);
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  offset = __float2half_rn(lo);
  scale = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f), kKv4MaxScale));
  const float s = __half2float(scale), o = __half2float(offset);
  if (!(s > 0.f)) return 0u;
  const float inv = __fdividef(1.f, s);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = __fsub_rn(v[i], o);
    float t = d * inv;
    // the reciprocal's product is off by a few units in the last place: only next to a border does the quotient itself decide
    if (fabsf(fabsf(t - rintf(t)) - 0.5f) < 1e-3f) t = __fdiv_rn(d, s);
    codes |= static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(rintf(t), 0.f), 15.f))) << (4 * i);
  }
  return codes;
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

// One CTA: the tokens of one block (consecutive positions of one page), one thread per token and 8 channels, looping over
// its share of the heads with the token's cosines and sines in registers. blockIdx.y < kv_parts: K and V heads; behind
// them, query heads.
template <int HD, int FMT>
__global__ void __launch_bounds__(2 * HD) kv_append_kernel(const KvAppendParams p) {
  constexpr int CH = HD / 8;
  __shared__ __align__(16) uint8_t image[image_bytes<HD, FMT>()];
  pdl_launch_dependents();
  pdl_wait();
  const KvBlock blk = p.blocks[blockIdx.x];
  const int i = threadIdx.x / CH, c = threadIdx.x % CH;
  const bool active = i < blk.n;
  const int tok = blk.tok0 + i;
  const bool first_half = c < CH / 2;
  float2 cs[8];
  const bool turn = p.rope != nullptr;
  if (turn && active) {
    const float4* r = reinterpret_cast<const float4*>(p.rope + static_cast<size_t>(tok) * (HD / 2) + (c * 8) % (HD / 2));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 f = __ldg(r + j);
      cs[2 * j] = make_float2(f.x, f.y);
      cs[2 * j + 1] = make_float2(f.z, f.w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[j] = make_float2(1.f, 0.f);
  }
  const bool bf16 = p.src_bf16 != 0;
  if (static_cast<int>(blockIdx.y) >= p.kv_parts) {
    const int part = blockIdx.y - p.kv_parts;
    const int h1 = min(p.n_q_heads, (part + 1) * p.q_heads_per_part);
    for (int h = part * p.q_heads_per_part; h < h1; ++h) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (active) raw = *reinterpret_cast<const uint4*>(p.q + tok * p.q_stride + h * HD + c * 8);
      float x[8];
      widen8(raw, bf16, x);
      turn8<HD>(x, raw, bf16, cs, first_half);
      if (active) *reinterpret_cast<uint4*>(p.q_out + tok * p.q_out_stride + h * HD + c * 8) = narrow8(x, bf16);
    }
    return;
  }
  const int pos = blk.pos0 + i;
  const int slot = pos % kPage;
  const int page = p.table[static_cast<size_t>(blk.seq) * p.max_pages_per_seq + blk.pos0 / kPage];
  const bool ok = debug_in_range(page >= 0 && page < p.num_pages && blk.pos0 / kPage < p.max_pages_per_seq, p.status);
  const bool whole = blk.n == kPage && FMT != CS_KV_FMT_16BIT;
  const int h1 = min(p.n_kv_heads, (static_cast<int>(blockIdx.y) + 1) * p.kv_heads_per_part);
  for (int h = blockIdx.y * p.kv_heads_per_part; h < h1; ++h) {
    uint4 rk = make_uint4(0, 0, 0, 0), rv = make_uint4(0, 0, 0, 0);
    if (active) {
      rk = *reinterpret_cast<const uint4*>(p.k + tok * p.k_stride + h * HD + c * 8);
      rv = *reinterpret_cast<const uint4*>(p.v + tok * p.v_stride + h * HD + c * 8);
    }
    float k[8], v[8];
    widen8(rk, bf16, k);
    widen8(rv, bf16, v);
    if (turn) turn8<HD>(k, rk, bf16, cs, first_half);
    const size_t ph = static_cast<size_t>(page) * p.n_kv_heads + h;
    if (FMT == CS_KV_FMT_16BIT) {
      // the 16-bit cache holds bf16 values in the fp16 encoding
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        k[j] = storable(__bfloat162float(__float2bfloat16_rn(k[j])), kF16Max);
        v[j] = storable(__bfloat162float(__float2bfloat16_rn(v[j])), kF16Max);
      }
      if (active && ok) {
        const size_t at = (ph * kPage + slot) * HD + c * 8;
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p.pool_k) + at) = narrow8(k, false);
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p.pool_v) + at) = narrow8(v, false);
      }
    } else if (FMT == CS_KV_FMT_INT4) {
      using L = Kv4<HD>;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        k[j] = storable(k[j], kF16Max);
        v[j] = storable(v[j], kF16Max);
      }
      __half ks, ko, vs, vo;
      const uint32_t kc = quantise8(k, ks, ko);
      const uint32_t vc = quantise8(v, vs, vo);
      const uint32_t vp = __shfl_xor_sync(0xffffffffu, vc, 1);
      uint8_t* block = p.pool_k + ph * L::kBlock;
      uint8_t* dst = whole ? image : block;
      if (active && ok) {
        // channel 2 a + b of the eight goes from nibble 2 a + b to nibble a + 4 b
        uint32_t word = 0;
#pragma unroll
        for (int a = 0; a < 4; ++a) word |= ((kc >> (8 * a)) & 15u) << (4 * a) | ((kc >> (8 * a + 4)) & 15u) << (4 * a + 16);
        *reinterpret_cast<uint32_t*>(dst + L::k_word(slot, c * 8)) = word;
        // V: tile c / 2; this thread holds its lower (c even) or upper eight channels and writes four of the eight bytes
        const uint32_t low = c & 1 ? vp : vc, high = c & 1 ? vc : vp;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int g = 4 * (c & 1) + j;
          dst[L::kVCodes + L::v_byte(slot, c >> 1, g)] = static_cast<uint8_t>((low >> (4 * g) & 15u) | (high >> (4 * g) & 15u) << 4);
        }
        if ((c & 7) == 0) {
          *reinterpret_cast<__half*>(dst + L::kKScale + L::k_param(slot, c / 8)) = ks;
          *reinterpret_cast<__half*>(dst + L::kKOffset + L::k_param(slot, c / 8)) = ko;
          *reinterpret_cast<__half*>(dst + L::v_scale(slot, c / 8)) = vs;
          *reinterpret_cast<__half*>(dst + L::v_offset(slot, c / 8)) = vo;
        }
      }
      if (whole) {
        __syncthreads();
        if (ok)
          for (int b = threadIdx.x; b < L::kBlock / 16; b += 2 * HD)
            reinterpret_cast<uint4*>(block)[b] = reinterpret_cast<const uint4*>(image)[b];
        __syncthreads();
      }
    } else {
      constexpr float most = FMT == CS_KV_FMT_E4M3 ? 448.f : 57344.f;
      uint2 kb;
      uint32_t w[2] = {0, 0};
      uint8_t vb[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j >> 2] |= static_cast<uint32_t>(fp8_of<FMT>(storable(k[j], most))) << (8 * (j & 3));
        vb[j] = fp8_of<FMT>(storable(v[j], most));
      }
      kb = make_uint2(w[0], w[1]);
      uint8_t* vt = p.pool_v + ph * kPage * HD;                  // V pages are kept transposed, [HD][16]
      uint8_t* dst = whole ? image : vt;
      if (active && ok) {
        *reinterpret_cast<uint2*>(p.pool_k + (ph * kPage + slot) * HD + c * 8) = kb;
#pragma unroll
        for (int j = 0; j < 8; ++j) dst[(c * 8 + j) * kPage + slot] = vb[j];
      }
      if (whole) {
        __syncthreads();
        if (ok)
          for (int b = threadIdx.x; b < HD; b += 2 * HD) reinterpret_cast<uint4*>(vt)[b] = reinterpret_cast<const uint4*>(image)[b];
        __syncthreads();
      }
    }
  }
}

template <int FMT>
__device__ __forceinline__ float fp8_value(uint8_t b) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw(b, FMT == CS_KV_FMT_E4M3 ? __NV_E4M3 : __NV_E5M2);
  return __half2float(__half(h));
}

// Rows listed by (sequence, position) out of the cache: one thread per row and 8 channels. A place outside the page table
// gives a row of zeros and raises the range bit of the status word.
template <int HD, int FMT>
__global__ void __launch_bounds__(2 * HD) kv_read_kernel(const KvReadParams p) {
  constexpr int CH = HD / 8;
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x * kPage + threadIdx.x / CH, c = threadIdx.x % CH;
  if (row >= p.T) return;
  const int seq = p.tok_seq[row], pos = p.tok_pos[row];
  int page = -1;
  if (seq >= 0 && seq < p.max_seqs && pos >= 0 && pos / kPage < p.max_pages_per_seq)
    page = p.table[static_cast<size_t>(seq) * p.max_pages_per_seq + pos / kPage];
  const bool ok = page >= 0 && page < p.num_pages;
  if (!ok && c == 0 && blockIdx.y == 0) atomicOr(p.status, kStatusRange);
  const int slot = pos & (kPage - 1);
  const int h1 = min(p.n_kv_heads, (static_cast<int>(blockIdx.y) + 1) * p.heads_per_part);
  for (int h = blockIdx.y * p.heads_per_part; h < h1; ++h) {
    float k[8] = {}, v[8] = {};
    if (ok) {
      const size_t ph = static_cast<size_t>(page) * p.n_kv_heads + h;
      if (FMT == CS_KV_FMT_16BIT) {
        const size_t at = (ph * kPage + slot) * HD + c * 8;
        widen8(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.pool_k) + at), false, k);
        widen8(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.pool_v) + at), false, v);
      } else if (FMT == CS_KV_FMT_INT4) {
        using L = Kv4<HD>;
        const uint8_t* b = p.pool_k + ph * L::kBlock;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(b + L::k_word(slot, c * 8));
        const float ks = __half2float(*reinterpret_cast<const __half*>(b + L::kKScale + L::k_param(slot, c / 8)));
        const float ko = __half2float(*reinterpret_cast<const __half*>(b + L::kKOffset + L::k_param(slot, c / 8)));
        const float vs = __half2float(*reinterpret_cast<const __half*>(b + L::v_scale(slot, c / 8)));
        const float vo = __half2float(*reinterpret_cast<const __half*>(b + L::v_offset(slot, c / 8)));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          k[j] = static_cast<float>(w >> (4 * (j / 2) + 16 * (j & 1)) & 15u) * ks + ko;
          const uint32_t byte = b[L::kVCodes + L::v_byte(slot, c >> 1, j)];
          v[j] = static_cast<float>(c & 1 ? byte >> 4 : byte & 15u) * vs + vo;
        }
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
    *reinterpret_cast<uint4*>(p.out_k + at) = narrow8(k, p.dst_bf16 != 0);
    *reinterpret_cast<uint4*>(p.out_v + at) = narrow8(v, p.dst_bf16 != 0);
  }
}

// Whole pages of the 4-bit cache as fp16 pages of one layer's scratch pool (the layout of the 16-bit cache): what the
// tensor-core attention of long steps reads. One CTA per (listed page, kv head).
template <int HD>
__global__ void __launch_bounds__(2 * HD) kv_expand_kernel(const uint8_t* __restrict__ pool, const int32_t* __restrict__ pages,
                                                          uint16_t* __restrict__ out_k, uint16_t* __restrict__ out_v,
                                                          int n_kv_heads, int num_pages, uint32_t* status) {
  using L = Kv4<HD>;
  constexpr int CH = HD / 8;
  __shared__ __align__(16) uint8_t b[L::kBlock];
  pdl_launch_dependents();
  pdl_wait();
  const int page = pages[blockIdx.x], h = blockIdx.y;
  if (!debug_in_range(page >= 0 && page < num_pages, status)) return;
  const size_t ph = static_cast<size_t>(page) * n_kv_heads + h;
  const uint4* src = reinterpret_cast<const uint4*>(pool + ph * L::kBlock);
  for (int i = threadIdx.x; i < L::kBlock / 16; i += 2 * HD) reinterpret_cast<uint4*>(b)[i] = __ldg(src + i);
  __syncthreads();
  const int slot = threadIdx.x / CH, c = threadIdx.x % CH;
  const uint32_t w = *reinterpret_cast<const uint32_t*>(b + L::k_word(slot, c * 8));
  const float ks = __half2float(*reinterpret_cast<const __half*>(b + L::kKScale + L::k_param(slot, c / 8)));
  const float ko = __half2float(*reinterpret_cast<const __half*>(b + L::kKOffset + L::k_param(slot, c / 8)));
  const float vs = __half2float(*reinterpret_cast<const __half*>(b + L::v_scale(slot, c / 8)));
  const float vo = __half2float(*reinterpret_cast<const __half*>(b + L::v_offset(slot, c / 8)));
  float k[8], v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    k[j] = static_cast<float>(w >> (4 * (j / 2) + 16 * (j & 1)) & 15u) * ks + ko;
    const uint32_t byte = b[L::kVCodes + L::v_byte(slot, c >> 1, j)];
    v[j] = static_cast<float>(c & 1 ? byte >> 4 : byte & 15u) * vs + vo;
  }
  const size_t at = (ph * kPage + slot) * HD + c * 8;
  *reinterpret_cast<uint4*>(out_k + at) = narrow8(k, false);
  *reinterpret_cast<uint4*>(out_v + at) = narrow8(v, false);
}

template <int HD>
cudaError_t append_hd(const KvAppendParams& p, int format, dim3 grid, cudaStream_t s) {
  switch (format) {
    case CS_KV_FMT_16BIT: return launch_pdl(kv_append_kernel<HD, CS_KV_FMT_16BIT>, grid, dim3(2 * HD), 0, s, p);
    case CS_KV_FMT_E4M3: return launch_pdl(kv_append_kernel<HD, CS_KV_FMT_E4M3>, grid, dim3(2 * HD), 0, s, p);
    case CS_KV_FMT_E5M2: return launch_pdl(kv_append_kernel<HD, CS_KV_FMT_E5M2>, grid, dim3(2 * HD), 0, s, p);
    case CS_KV_FMT_INT4: return launch_pdl(kv_append_kernel<HD, CS_KV_FMT_INT4>, grid, dim3(2 * HD), 0, s, p);
    default: return cudaErrorInvalidValue;
  }
}

template <int HD>
cudaError_t read_hd(const KvReadParams& p, int format, dim3 grid, cudaStream_t s) {
  switch (format) {
    case CS_KV_FMT_16BIT: return launch_pdl(kv_read_kernel<HD, CS_KV_FMT_16BIT>, grid, dim3(2 * HD), 0, s, p);
    case CS_KV_FMT_E4M3: return launch_pdl(kv_read_kernel<HD, CS_KV_FMT_E4M3>, grid, dim3(2 * HD), 0, s, p);
    case CS_KV_FMT_E5M2: return launch_pdl(kv_read_kernel<HD, CS_KV_FMT_E5M2>, grid, dim3(2 * HD), 0, s, p);
    case CS_KV_FMT_INT4: return launch_pdl(kv_read_kernel<HD, CS_KV_FMT_INT4>, grid, dim3(2 * HD), 0, s, p);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace

cudaError_t launch_kv_append(KvAppendParams p, int format, int hd, int n_blocks, cudaStream_t s) {
  if (n_blocks <= 0) return cudaSuccess;
  // few blocks: one head per CTA, for latency; many: several, which read the token's cosines and sines once
  int per = 1;
  while (per < 4 && static_cast<long>(n_blocks) * ((p.n_kv_heads + 2 * per - 1) / (2 * per)) >= 8L * kNumSMs) per *= 2;
  p.kv_heads_per_part = per;
  p.kv_parts = (p.n_kv_heads + per - 1) / per;
  p.q_heads_per_part = 2 * per;
  const int q_parts = p.q ? (p.n_q_heads + 2 * per - 1) / (2 * per) : 0;
  const dim3 grid(n_blocks, p.kv_parts + q_parts);
  const cudaError_t e = hd == 128 ? append_hd<128>(p, format, grid, s) : append_hd<64>(p, format, grid, s);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv_read(KvReadParams p, int format, int hd, cudaStream_t s) {
  if (p.T <= 0) return cudaSuccess;
  const int blocks = (p.T + kPage - 1) / kPage;
  p.heads_per_part = 1;
  const dim3 grid(blocks, p.n_kv_heads);
  const cudaError_t e = hd == 128 ? read_hd<128>(p, format, grid, s) : read_hd<64>(p, format, grid, s);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv_expand(const uint8_t* pool, const int32_t* pages, int n_pages, uint16_t* out_k, uint16_t* out_v,
                             int n_kv_heads, int hd, int num_pages, uint32_t* status, cudaStream_t s) {
  if (n_pages <= 0) return cudaSuccess;
  const dim3 grid(n_pages, n_kv_heads), block(2 * hd);
  const cudaError_t e =
      hd == 128 ? launch_pdl(kv_expand_kernel<128>, grid, block, 0, s, pool, pages, out_k, out_v, n_kv_heads, num_pages, status)
                : launch_pdl(kv_expand_kernel<64>, grid, block, 0, s, pool, pages, out_k, out_v, n_kv_heads, num_pages, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace cs
