// Attention over a cache held in 4 bits (layout: kv4.cuh), for one new token or a few tens of them per step, grouped query
// heads, ragged contexts.
//
// Mathematics. A cached key is k_d = s c_d + o with one (s, o) per 64-channel group, so
//     q . k = sum_groups s (sum_d q_d c_d) + o (sum_d q_d),         out_d = sum_j p_j (s_j c_jd + o_j)
// and the products run over the integer codes, which are exact in fp16: scales multiply the fp32 sums of a group (keys) or
// the codes in registers (values), offsets go through one small product each.
//
// Shape. The keys are the rows of the products and the query rows (token, head of the group) their columns: 16 keys x 8
// query rows x 16 channels per instruction, so that a decode step's few query rows (one token, up to 8 heads per kv head)
// cost half of what the usual orientation, with its 16-row query tile, would. S^T = K Q^T leaves a key's scores in one
// lane pair of columns; P^T turns into the operand of O^T = V^T P^T by two 8 x 8 register transposes.
//
// Bound. Reading the cache: HD / 2 + 4 HD / 64 bytes per row of K or V. Every warp streams whole (page, kv head) blocks with
// asynchronous copies, two in flight; nothing waits on another CTA. At the copy bandwidth an SM has ~100 cycles per block,
// some 400 issue slots over its four schedulers, against ~260 instructions per block (8 query rows, HD = 128): what follows
// counts instructions. Codes become fp16 operands with one mask and one shift per pair (no conversion instruction): a
// nibble in the mantissa of a power of two, 64 + c, whose 64 is taken back by the accumulator's start value (keys), or
// 64 + c / 16 and 4 + c / 16, which one fused multiply-add turns into s c / 16 exactly before rounding (values).
// A piece of a long context leaves (max, sum, O) in fp32 and a second kernel joins the pieces in a fixed order.
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "kv4.cuh"

namespace cs {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = 4;
constexpr int kPage = 16;
constexpr int kStages = 3;
constexpr float kNoMax = -1.0e30f;
// The running maximum is raised only when a score passes it by this much (powers of two): probabilities reach 2^8, which
// fp16 and the fp32 sums hold with their full relative precision, and most pages leave the accumulators alone.
constexpr float kMaxSlack = 8.f;

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// D (16 x 8, fp32) = A (16 x 16, fp16, row) * B (16 x 8, fp16, col) + C
__device__ __forceinline__ void mma_k16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1,
                                        float c2, float c3) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void mma_k16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  mma_k16(d, a, b0, b1, d[0], d[1], d[2], d[3]);
}
// D (16 x 8, fp32) = A (16 x 8, fp16, row) * B (8 x 8, fp16, col)
__device__ __forceinline__ void mma_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%7, %7, %7, %7};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a0), "r"(a1), "r"(b0), "f"(0.f));
}
// 8 x 8 matrix of 16-bit elements spread over the warp, transposed
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t hmul2_u(uint32_t a, uint32_t b) {
  __half2 r = __hmul2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t hfma2_u(uint32_t a, uint32_t b, uint32_t c) {
  __half2 r = __hfma2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b), *reinterpret_cast<__half2*>(&c));
  return *reinterpret_cast<uint32_t*>(&r);
}
// nibbles 0 and 4 of w: 64 + c / 16;  nibbles 1 and 5: 4 + c / 16, or 64 + c when placed under the exponent of 64
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return (w & 0x000F000Fu) | 0x54005400u; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return (w & 0x00F000F0u) | 0x44004400u; }
__device__ __forceinline__ uint32_t whole_codes(uint32_t w) { return (w & 0x00F000F0u) | 0x54005400u; }

// Eight 16-bit values as fp16: bf16 sources are re-encoded (exact for magnitudes in [2^-14, 65504]).
__device__ __forceinline__ uint4 as_f16(uint4 v, bool bf16) {
  return bf16 ? make_uint4(bf16x2_to_f16x2(v.x), bf16x2_to_f16x2(v.y), bf16x2_to_f16x2(v.z), bf16x2_to_f16x2(v.w)) : v;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

__device__ __forceinline__ void store_out(const Attn4Params& p, size_t at, float v) {
  if (p.out_bf16) reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
  else reinterpret_cast<__half*>(p.out)[at] = __float2half_rn(v);
}

template <int HD, int NT>
struct Smem4 {
  static constexpr int kWarp = kStages * Kv4<HD>::kBlock;
  static constexpr int kStagesBytes = kWarps * kWarp;
  static constexpr int kPad = HD + 4;                                  // row stride of the partial results, in floats
  static constexpr int kPartBytes = kWarps * 8 * NT * kPad * 4;
  static constexpr int kStatBytes = kWarps * 8 * NT * 2 * 4;
  static constexpr int kUnion = kStagesBytes > kPartBytes + kStatBytes ? kStagesBytes : kPartBytes + kStatBytes;
  // 32 query rows: the query operands do not fit the registers beside the accumulators
  static constexpr int kQBytes = NT > 2 ? 8 * NT * HD * 2 : 0;
  static constexpr int kTotal = kUnion + kQBytes;
  static_assert(kWarp >= kPage * HD * 2, "a page of own values must fit in one warp's stages");
};

// NT = number of 8-row tiles of query rows (1, 2 or 4).
template <int HD, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 4 : NT == 2 ? 3 : 2)
attention_4bit_kernel(const Attn4Params p, const AttnItem* __restrict__ items) {
  using L = Kv4<HD>;
  using S = Smem4<HD, NT>;
  constexpr int NG = L::kGroups;            // channel groups
  constexpr int MT = HD / 16;               // 16-channel tiles of the output
  constexpr bool kQInRegs = NT <= 2;
  extern __shared__ __align__(128) uint8_t smem[];
  pdl_launch_dependents();
  const AttnItem it = items[blockIdx.x];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q = lane & 3;
  const int G = p.n_q_heads / p.n_kv_heads;
  const int row0 = it.q_tok0;                             // first query row (token * G + head in group) of this tile
  const int R = min(8 * NT, it.n_new * G - row0);         // query rows in use
  uint8_t* my = smem + warp * S::kWarp;
  const uint32_t my_u = smem_u32(my);
  const int32_t* table = p.page_table + static_cast<size_t>(it.seq) * p.max_pages_per_seq;
  const int cached_pages = it.pad[1];
  const size_t page_stride = static_cast<size_t>(p.n_kv_heads) * L::kBlock;
  const uint8_t* pool_h = p.pool + static_cast<size_t>(it.kv_head) * L::kBlock;
  const int end_cached = min(it.tile_end, cached_pages);

  auto fetch = [&](int32_t id, int stage) {
    if (!debug_in_range(id >= 0 && id < p.num_pages, p.status)) id = 0;
    const uint8_t* src = pool_h + static_cast<size_t>(id) * page_stride + lane * 16;
    const uint32_t dst = my_u + stage * L::kBlock + lane * 16;
#pragma unroll
    for (int c = 0; c < L::kBlock / 512; ++c) cp_async_16(dst + c * 512, src + c * 512);
    if (lane < (L::kBlock % 512) / 16) cp_async_16(dst + L::kBlock / 512 * 512, src + L::kBlock / 512 * 512);
  };
  const int pg0 = it.tile_begin + warp;
  // Where nothing that precedes this kernel on the stream writes the cache (the verification pass), the first pages are
  // requested before the wait; a caller who has just appended waits first.
  if (!p.cache_is_settled) pdl_wait();
  int32_t ids[kStages];
#pragma unroll
  for (int st = 0; st < kStages; ++st) ids[st] = pg0 + st * kWarps < end_cached ? __ldg(table + pg0 + st * kWarps) : 0;
#pragma unroll
  for (int st = 0; st < kStages - 1; ++st) {
    if (pg0 + st * kWarps < end_cached) fetch(ids[st], st);
    cp_async_commit();
  }
  int32_t id_ahead = ids[kStages - 1];
  if (p.cache_is_settled) pdl_wait();

  // Query operands. Lane (g, q) holds, for each group and each of the two words of a key row's chunk, the eight channels
  // 64 group + 16 q + 8 w .. + 7 of query row g of a tile: two k-steps of the score product.
  uint4 qr[kQInRegs ? NT : 1][NG][2];
  uint32_t qoff[NT];           // operand of the offsets' product: sums of q over (half a group), high and low parts
  float qneg[NT][NG][2];       // -64 sum_group q of query rows 2 q and 2 q + 1: the accumulators' start values
  uint8_t* q_s = smem + S::kUnion;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = nt * 8 + g;
    uint4 v[NG][2];
    float sum[NG];
    const int t = (row0 + r) / G, hq = (row0 + r) % G;
#pragma unroll
    for (int grp = 0; grp < NG; ++grp) {
      sum[grp] = 0.f;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        v[grp][w] = make_uint4(0, 0, 0, 0);
        if (r < R)
          v[grp][w] = as_f16(*reinterpret_cast<const uint4*>(p.q + (it.tok0 + t) * p.q_stride + (it.kv_head * G + hq) * HD +
                                                             grp * 64 + q * 16 + w * 8), p.in_bf16 != 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = unpack_f16x2(word(v[grp][w], i));
          sum[grp] += f.x + f.y;
        }
        if (kQInRegs) qr[nt][grp][w] = v[grp][w];
        else if (warp == 0) *reinterpret_cast<uint4*>(q_s + ((nt * NG + grp) * 2 + w) * 512 + lane * 16) = v[grp][w];
      }
      sum[grp] += __shfl_xor_sync(0xffffffffu, sum[grp], 1);     // lanes q = 0, 1 and q = 2, 3: half a group each
    }
    // A half group's sum in two fp16 parts (22 bits); the four lanes of a row give the four slots of the k = 8 product.
    float part[2];
#pragma unroll
    for (int grp = 0; grp < 2; ++grp) {
      const float f = grp < NG ? sum[grp < NG ? grp : 0] : 0.f;
      const float hi = __half2float(__float2half_rn(f));
      part[grp] = q & 1 ? f - hi : hi;
    }
    qoff[nt] = pack_f16x2(part[0], part[1]);
#pragma unroll
    for (int grp = 0; grp < NG; ++grp) {
      const float total = sum[grp] + __shfl_xor_sync(0xffffffffu, sum[grp], 2);
      qneg[nt][grp][0] = -64.f * __shfl_sync(0xffffffffu, total, 8 * q);
      qneg[nt][grp][1] = -64.f * __shfl_sync(0xffffffffu, total, 8 * q + 4);
    }
  }
  if (!kQInRegs) __syncthreads();
  auto q_words = [&](int nt, int grp, int w) -> uint4 {
    if (kQInRegs) return qr[kQInRegs ? nt : 0][grp][w];
    return *reinterpret_cast<const uint4*>(q_s + ((nt * NG + grp) * 2 + w) * 512 + lane * 16);
  };

  float o[NT][MT][4];          // O^T / 16 without the offsets' share: channels 16 mt + g, + 8; query rows 2 q, 2 q + 1
  float oo[NT][4];             // sum_j p_j o_j: of group g & 1 (first two) and of the other group
  float m_run[NT][2], l_run[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m_run[nt][0] = m_run[nt][1] = kNoMax;
    l_run[nt][0] = l_run[nt][1] = 0.f;
    oo[nt][0] = oo[nt][1] = oo[nt][2] = oo[nt][3] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
  }

  // Scores of 16 keys (s[nt]: keys g, g + 8 x query rows 2 q, 2 q + 1) -> probabilities as the operand of the output product.
  auto softmax = [&](float (&s)[NT][4], uint32_t (&pb)[NT][2]) {
    bool raise = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float a = fmaxf(s[nt][0], s[nt][2]), b = fmaxf(s[nt][1], s[nt][3]);
      raise = raise || a * p.scale_log2e > m_run[nt][0] + kMaxSlack || b * p.scale_log2e > m_run[nt][1] + kMaxSlack;
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(s[nt][e], s[nt][e + 2]) * p.scale_log2e;
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const float m_new = fmaxf(m_run[nt][e], mx);
          const float corr = fast_exp2(m_run[nt][e] - m_new);
          m_run[nt][e] = m_new;
          l_run[nt][e] *= corr;
          oo[nt][e] *= corr;
          oo[nt][e + 2] *= corr;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            o[nt][mt][e] *= corr;
            o[nt][mt][e + 2] *= corr;
          }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][e] = fast_exp2(fmaf(s[nt][e], p.scale_log2e, -m_run[nt][e & 1]));
      l_run[nt][0] += s[nt][0] + s[nt][2];
      l_run[nt][1] += s[nt][1] + s[nt][3];
      pb[nt][0] = transpose8x8(pack_f16x2(s[nt][0], s[nt][1]));
      pb[nt][1] = transpose8x8(pack_f16x2(s[nt][2], s[nt][3]));
    }
  };
  // Keys key0 .. key0 + 15 against the last key that the rows of token t see, base + t: masked scores are -inf.
  const int t_min = row0 / G;
  auto mask = [&](float (&s)[NT][4], int key0, int base, int per_token) {
    if (key0 + kPage - 1 <= base + per_token * t_min) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = (row0 + nt * 8 + 2 * q + (e & 1)) / G;
        if (key0 + g + (e >> 1) * 8 > base + per_token * t) s[nt][e] = -INFINITY;
      }
  };

  auto cached_page = [&](const uint8_t* b, int key0) {
    float acc[NT][NG][4];
    uint32_t kw[2][2 * NG];
    if (NG == 2) {
      *reinterpret_cast<uint4*>(kw[0]) = *reinterpret_cast<const uint4*>(b + g * (HD / 2) + q * (HD / 8));
      *reinterpret_cast<uint4*>(kw[1]) = *reinterpret_cast<const uint4*>(b + (g + 8) * (HD / 2) + q * (HD / 8));
    } else {
      *reinterpret_cast<uint2*>(kw[0]) = *reinterpret_cast<const uint2*>(b + g * (HD / 2) + q * (HD / 8));
      *reinterpret_cast<uint2*>(kw[1]) = *reinterpret_cast<const uint2*>(b + (g + 8) * (HD / 2) + q * (HD / 8));
    }
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int grp = 0; grp < NG; ++grp) {
        const uint32_t wa = kw[0][2 * grp + w], wb = kw[1][2 * grp + w];
        const uint32_t a0[4] = {whole_codes(wa << 4), whole_codes(wb << 4), whole_codes(wa), whole_codes(wb)};
        const uint32_t a1[4] = {whole_codes(wa >> 4), whole_codes(wb >> 4), whole_codes(wa >> 8), whole_codes(wb >> 8)};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 qv = q_words(nt, grp, w);
          if (w == 0)
            mma_k16(acc[nt][grp], a0, qv.x, qv.y, qneg[nt][grp][0], qneg[nt][grp][1], qneg[nt][grp][0], qneg[nt][grp][1]);
          else
            mma_k16(acc[nt][grp], a0, qv.x, qv.y);
          mma_k16(acc[nt][grp], a1, qv.z, qv.w);
        }
      }
    // scales (fp32) and offsets of keys g and g + 8
    float sc[2][NG];
    uint32_t off[2];
    if (NG == 2) {
      const uint2 s2 = *reinterpret_cast<const uint2*>(b + L::kKScale + g * 8);
      const uint2 o2 = *reinterpret_cast<const uint2*>(b + L::kKOffset + g * 8);
      const float2 f0 = unpack_f16x2(s2.x), f1 = unpack_f16x2(s2.y);
      sc[0][0] = f0.x; sc[0][NG - 1] = f0.y; sc[1][0] = f1.x; sc[1][NG - 1] = f1.y;
      off[0] = o2.x; off[1] = o2.y;
    } else {
      const float2 f = unpack_f16x2(*reinterpret_cast<const uint32_t*>(b + L::kKScale + g * 4));
      const uint32_t o1 = *reinterpret_cast<const uint32_t*>(b + L::kKOffset + g * 4);
      sc[0][0] = f.x; sc[1][0] = f.y;
      off[0] = __byte_perm(o1, o1, 0x1010); off[1] = __byte_perm(o1, o1, 0x3232);
    }
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mma_k8(s[nt], off[0], off[1], qoff[nt]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int grp = 0; grp < NG; ++grp) s[nt][e] = fmaf(sc[e >> 1][grp], acc[nt][grp][e], s[nt][e]);
    }
    mask(s, key0, it.ctx - (p.given ? 1 : 0), p.given ? 0 : 1);
    uint32_t pb[NT][2];
    softmax(s, pb);

    // values: scales of keys (2 q, 2 q + 1) and (2 q + 8, 2 q + 9) per group, and what takes the 64 and the 4 back
    uint32_t vs[2 * NG], n64[2 * NG], n4[2 * NG];
    if (NG == 2) *reinterpret_cast<uint4*>(vs) = *reinterpret_cast<const uint4*>(b + L::kVScale + q * 16);
    else *reinterpret_cast<uint2*>(vs) = *reinterpret_cast<const uint2*>(b + L::kVScale + q * 8);
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) {
      n64[i] = hmul2_u(vs[i], 0xD400D400u);       // -64
      n4[i] = hmul2_u(vs[i], 0xC400C400u);        // -4
    }
    const uint8_t* vb = b + L::kVCodes + L::v_chunk(g, q) * 16;
#pragma unroll
    for (int half = 0; half < NG; ++half) {
      const uint4 vw = *reinterpret_cast<const uint4*>(vb + half * 512);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = word(vw, i), w8 = w >> 8;
        const uint32_t a[4] = {hfma2_u(low_codes(w), vs[2 * half], n64[2 * half]),
                               hfma2_u(high_codes(w), vs[2 * half], n4[2 * half]),
                               hfma2_u(low_codes(w8), vs[2 * half + 1], n64[2 * half + 1]),
                               hfma2_u(high_codes(w8), vs[2 * half + 1], n4[2 * half + 1])};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_k16(o[nt][4 * half + i], a, pb[nt][0], pb[nt][1]);
      }
    }
    uint32_t ao[4];
    {
      const uint2 x = *reinterpret_cast<const uint2*>(b + L::kVOffset + (q * NG + (NG == 2 ? g & 1 : 0)) * 8);
      const uint2 y = *reinterpret_cast<const uint2*>(b + L::kVOffset + (q * NG + (NG == 2 ? (g & 1) ^ 1 : 0)) * 8);
      ao[0] = x.x; ao[1] = y.x; ao[2] = x.y; ao[3] = y.y;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mma_k16(oo[nt], ao, pb[nt][0], pb[nt][1]);
  };

  // A page of the step's own keys and values, given as rows in fp16 or bf16: K operands straight from global memory, V through
  // this warp's (drained) stages and transposing loads. V is divided by 16, as the cached values are.
  auto own_page = [&](int key0) {
    cp_async_wait<0>();
    __syncwarp();
    constexpr int CH = HD / 8;
    for (int c = lane; c < kPage * CH; c += 32) {
      const int key = c / CH, ch = c % CH;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (key0 + key < it.n_new)
        v = as_f16(*reinterpret_cast<const uint4*>(p.v_new + (it.tok0 + key0 + key) * p.kv_stride + it.kv_head * HD + ch * 8),
                   p.in_bf16 != 0);
      v = make_uint4(hmul2_u(v.x, 0x2C002C00u), hmul2_u(v.y, 0x2C002C00u), hmul2_u(v.z, 0x2C002C00u), hmul2_u(v.w, 0x2C002C00u));
      *reinterpret_cast<uint4*>(my + key * HD * 2 + ((ch ^ (key & 7)) << 4)) = v;
    }
    __syncwarp();
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
    for (int grp = 0; grp < NG; ++grp)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint4 x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int key = key0 + g + 8 * j;
          x[j] = make_uint4(0, 0, 0, 0);
          if (key < it.n_new)
            x[j] = as_f16(*reinterpret_cast<const uint4*>(p.k_new + (it.tok0 + key) * p.kv_stride + it.kv_head * HD + grp * 64 +
                                                          q * 16 + w * 8), p.in_bf16 != 0);
        }
        const uint32_t a0[4] = {x[0].x, x[1].x, x[0].y, x[1].y}, a1[4] = {x[0].z, x[1].z, x[0].w, x[1].w};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 qv = q_words(nt, grp, w);
          mma_k16(s[nt], a0, qv.x, qv.y);
          mma_k16(s[nt], a1, qv.z, qv.w);
        }
      }
    mask(s, key0, 0, 1);
    uint32_t pb[NT][2];
    softmax(s, pb);
    // matrices of an operand tile: channels 0-7 / 8-15 x keys 0-7, then x keys 8-15
    const int key = (lane & 7) + (lane >> 4) * 8, up = (lane >> 3) & 1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      uint32_t a[4];
      ldmatrix_x4_trans(a, my_u + key * HD * 2 + (((2 * mt + up) ^ (key & 7)) << 4));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_k16(o[nt][mt], a, pb[nt][0], pb[nt][1]);
    }
    __syncwarp();
  };

  int pg = pg0;
  int stage = 0, ahead_stage = kStages - 1;
  for (; pg < end_cached; pg += kWarps) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    // the stage read in the previous round is free: request the page kStages - 1 rounds ahead
    const int ahead = pg + (kStages - 1) * kWarps;
    if (ahead < end_cached) fetch(id_ahead, ahead_stage);
    cp_async_commit();
    if (ahead + kWarps < end_cached) id_ahead = __ldg(table + ahead + kWarps);
    cached_page(my + stage * L::kBlock, pg * kPage);
    stage = stage == kStages - 1 ? 0 : stage + 1;
    ahead_stage = ahead_stage == kStages - 1 ? 0 : ahead_stage + 1;
  }
  for (; pg < it.tile_end; pg += kWarps) own_page((pg - cached_pages) * kPage);
  cp_async_wait<0>();
  __syncthreads();

  // ------------------------------------------------------------------ the warps' results, joined in warp order
  float* po = reinterpret_cast<float*>(smem);                            // [warp][8 NT rows][HD + 4]
  float* pml = reinterpret_cast<float*>(smem + S::kPartBytes);           // [warp][8 NT rows][2]
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = l_run[nt][e];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      const int r = nt * 8 + 2 * q + e;
      if (g == 0) {
        pml[(warp * 8 * NT + r) * 2] = m_run[nt][e];
        pml[(warp * 8 * NT + r) * 2 + 1] = l;
      }
      float* dst = po + (warp * 8 * NT + r) * S::kPad + g;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        // the group of this tile's channels: mt / 4; this lane's first pair of offset sums belongs to group g & 1
        const float add = NG == 1 || (mt / 4) == (g & 1) ? oo[nt][e] : oo[nt][e + 2];
        dst[mt * 16] = fmaf(16.f, o[nt][mt][e], add);
        dst[mt * 16 + 8] = fmaf(16.f, o[nt][mt][e + 2], add);
      }
    }
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < R * HD; idx += kThreads) {
    const int r = idx / HD, d = idx % HD;
    float M = kNoMax;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, pml[(w * 8 * NT + r) * 2]);
    float acc = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = fast_exp2(pml[(w * 8 * NT + r) * 2] - M);
      acc += f * po[(w * 8 * NT + r) * S::kPad + d];
      sum += f * pml[(w * 8 * NT + r) * 2 + 1];
    }
    if (it.n_splits == 1) {
      const int t = (row0 + r) / G, hq = (row0 + r) % G;
      store_out(p, (it.tok0 + t) * p.out_stride + (it.kv_head * G + hq) * HD + d, sum > 0.f ? acc / sum : 0.f);
    } else {
      p.part_o[(static_cast<size_t>(it.slot) * 32 + r) * HD + d] = acc;
      if (d == 0) {
        p.part_ml[(static_cast<size_t>(it.slot) * 32 + r) * 2] = M;
        p.part_ml[(static_cast<size_t>(it.slot) * 32 + r) * 2 + 1] = sum;
      }
    }
  }
}

// Pieces of one (step, kv head, row tile) -> output. One CTA per work item and 8 query rows; only the first piece does anything.
template <int HD>
__global__ void __launch_bounds__(HD) attention_4bit_merge_kernel(const Attn4Params p, const AttnItem* __restrict__ items, int tile) {
  pdl_launch_dependents();
  pdl_wait();
  const AttnItem it = items[blockIdx.x];
  if (it.n_splits <= 1 || it.slot != it.slot0) return;
  const int G = p.n_q_heads / p.n_kv_heads;
  const int R = min(tile, it.n_new * G - it.q_tok0);
  const int d = threadIdx.x;
  for (int r = blockIdx.y; r < R; r += gridDim.y) {
    float M = kNoMax;
    for (int s = 0; s < it.n_splits; ++s) M = fmaxf(M, p.part_ml[(static_cast<size_t>(it.slot0 + s) * 32 + r) * 2]);
    float acc = 0.f, sum = 0.f;
    for (int s = 0; s < it.n_splits; ++s) {
      const size_t base = static_cast<size_t>(it.slot0 + s) * 32 + r;
      const float f = fast_exp2(p.part_ml[base * 2] - M);
      acc += f * p.part_o[base * HD + d];
      sum += f * p.part_ml[base * 2 + 1];
    }
    const int t = (it.q_tok0 + r) / G, hq = (it.q_tok0 + r) % G;
    store_out(p, (it.tok0 + t) * p.out_stride + (it.kv_head * G + hq) * HD + d, sum > 0.f ? acc / sum : 0.f);
  }
}

template <int HD, int NT>
cudaError_t launch_4bit(const Attn4Params& p, const AttnItem* items, int n_items, bool any_split, cudaStream_t s) {
  static std::atomic<uint64_t> smem_opted{0};
  if (cudaError_t e = opt_in_dynamic_smem(attention_4bit_kernel<HD, NT>, Smem4<HD, NT>::kTotal, smem_opted); e != cudaSuccess)
    return e;
  cudaError_t e = launch_pdl(attention_4bit_kernel<HD, NT>, dim3(n_items), dim3(kThreads), Smem4<HD, NT>::kTotal, s, p, items);
  count_launch();
  if (e != cudaSuccess || !any_split) return e != cudaSuccess ? e : cudaGetLastError();
  e = launch_pdl(attention_4bit_merge_kernel<HD>, dim3(n_items, NT), dim3(HD), 0, s, p, items, 8 * NT);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// 8, 16 or 32 query rows per work item: the smallest tile that takes the batch's longest step whole, so that no step reads
// its context twice; longer steps are cut into tiles of 32.
int attention_4bit_row_tile(int max_rows) { return max_rows <= 8 ? 8 : max_rows <= 16 ? 16 : 32; }

cudaError_t launch_attention_4bit(const Attn4Params& p, const AttnItem* items, int n_items, int row_tile, bool any_split,
                                  cudaStream_t s) {
  if (n_items <= 0) return cudaSuccess;
  if (p.head_dim == 128)
    return row_tile == 8    ? launch_4bit<128, 1>(p, items, n_items, any_split, s)
           : row_tile == 16 ? launch_4bit<128, 2>(p, items, n_items, any_split, s)
                            : launch_4bit<128, 4>(p, items, n_items, any_split, s);
  if (p.head_dim == 64)
    return row_tile == 8    ? launch_4bit<64, 1>(p, items, n_items, any_split, s)
           : row_tile == 16 ? launch_4bit<64, 2>(p, items, n_items, any_split, s)
                            : launch_4bit<64, 4>(p, items, n_items, any_split, s);
  return cudaErrorInvalidValue;
}

}  // namespace cs
