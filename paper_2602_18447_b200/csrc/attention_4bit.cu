// Attention over a cache held in 4 bits (layout: kv4.cuh), for one new token or a few tens of them per step, grouped query
// heads, ragged contexts.
//
// Mathematics. A cached key is k_d = s c_d + o with one (s, o) per 64-channel group, so
//     q . k = sum_groups s (sum_d q_d c_d) + o (sum_d q_d),         out_d = sum_j p_j (s_j c_jd + o_j)
// and the products run over the integer codes, which are exact in fp16: scales multiply the fp32 sums of a group (keys) or
// the probabilities (values), offsets go through one small product each. Value codes are centred, c - 8, which halves the
// rounding of p s: it then weighs a value's distance from the middle of its group's range, not from its end.
//
// Shape. The keys are the rows of the products and the query rows (token, head of the group) their columns: 16 keys x 8
// query rows x 16 channels per instruction, so that a decode step's few query rows (one token, up to 8 heads per kv head)
// cost half of what the usual orientation, with its 16-row query tile, would. S^T = K Q^T leaves a key's scores in one
// lane pair of columns; P^T turns into the operand of O^T = V^T P^T by two 8 x 8 register transposes.
//
// Bound. Reading the cache: HD / 2 + 4 HD / 64 bytes per row of K or V. Every warp streams whole (page, kv head) blocks with
// asynchronous copies, two pages at a time and two such rounds ahead; nothing waits on another CTA but the CTAs of a cluster at
// their end. At the copy bandwidth an SM has ~100 cycles per block, some 400 issue slots over its four schedulers, against 255
// instructions per block at 8 query rows (336 at 16), HD = 128: what follows counts instructions. Codes become fp16 operands without
// a conversion instruction: a nibble in the mantissa of a power of two, 64 + c or 1024 + c. The 64 of half of a key's channels is
// taken back by the product that adds the offsets,
//     q . k = sum_groups s (sum_d q_d h_d) + o (sum_d q_d) - 64 s (sum over those channels of q_d),
// whose operands are the offsets and scales as they are stored; one packed addition makes c (keys) or c - 8 (values) of the
// others. The product that sums the values' offsets has rows of ones besides, which sum the probabilities.
// Measured on 64 contexts of 2 K to 8 K keys x 8 heads of 128 (0.37 GB): one token each (2 query rows per kv head) 69.2 us, 5.4 TB/s,
// 0.82 of the copy bandwidth; 5 to 8 tokens (16 rows) 110 us, 0.52, where the accumulators leave 12 warps on an SM and the products'
// latencies show (tensor pipe 40 % busy, 1.87 instructions a cycle); 17 to 96 rows some 90 us for every 16 rows begun, which read and
// unpack the pages anew. Two warps that share pages and split the channels (16 warps) were slower, 126 us where this form took 109:
// a third more instructions a block with the exchange of the probabilities.
//
// Pieces of a context are joined in their order. Where a few per context fill the machine, they are the CTAs of one cluster, which
// read one another's (max, sum, O) through shared memory: one launch. Else a piece leaves them in global memory and a second kernel,
// one CTA per query row, joins them. (Joining by the last piece to finish saves that launch but takes longer, even for few pieces:
// the fence, the counter and the reads follow one another at the end of the chain, while the second kernel's start overlaps this
// one. One token on 512 keys 7.9 us against 6.0, 16 sequences of up to 2048 10.7 against 9.2.)
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "kv4.cuh"

namespace cs {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = 4;
constexpr int kPage = 16;
constexpr int kStages = 3;              // of two pages each, per warp
constexpr float kNoMax = -1.0e30f;
constexpr uint32_t kOnes = 0x3C003C00u;      // two fp16 ones
// Probabilities are taken against a reference below the running maximum, so that the largest is 2^kHeadroom when the reference
// is set and up to 2^kRaise before it is raised: most pages leave the accumulators alone, small probabilities keep fp16's
// relative precision down to 2^-16 of the largest, and p s stays in fp16's range for every scale (kKv4MaxScale).
constexpr float kHeadroom = 2.f, kRaise = 6.f;
// Value scales are taken times up to 2^15 (as fp16 pairs: the factor, and the largest scale that may be taken times it).
constexpr int kMaxUp = 15;
constexpr uint32_t k2Max = 0x78007800u, kMostAt2Max = 0x27FF27FFu;

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// D (16 x 8, fp32) += A (16 x 16, fp16, row) * B (16 x 8, fp16, col)
__device__ __forceinline__ void mma_k16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same without an addend
__device__ __forceinline__ void mma_k16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// 8 x 8 matrix of 16-bit elements spread over the warp, transposed
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
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
__device__ __forceinline__ uint32_t hmax2_u(uint32_t a, uint32_t b) {
  __half2 r = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t hadd2_u(uint32_t a, uint32_t b) {
  __half2 r = __hadd2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
// (w & mask) | bits as one instruction (the compiler makes two of the expression)
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
  return r;
}
// nibbles 1 and 5 of w as 64 + c
__device__ __forceinline__ uint32_t codes64(uint32_t w) { return and_or(w, 0x00F000F0u, 0x54005400u); }
// c of nibbles 0 and 4 (1024 + c - 1024), exact
__device__ __forceinline__ uint32_t codes_low(uint32_t w) { return hadd2_u(and_or(w, 0x000F000Fu, 0x64006400u), 0xE400E400u); }
// c - 8 of nibbles 0 and 4 (1024 + c - 1032) and of nibbles 1 and 5 (64 + c - 72), exact
__device__ __forceinline__ uint32_t centred_low(uint32_t w) { return hadd2_u(and_or(w, 0x000F000Fu, 0x64006400u), 0xE408E408u); }
__device__ __forceinline__ uint32_t centred_high(uint32_t w) { return hadd2_u(codes64(w), 0xD480D480u); }

// Eight 16-bit values as fp16: bf16 sources are re-encoded (exact for magnitudes in [2^-14, 65504]).
__device__ __forceinline__ uint4 as_f16(uint4 v, bool bf16) {
  return bf16 ? make_uint4(bf16x2_to_f16x2(v.x), bf16x2_to_f16x2(v.y), bf16x2_to_f16x2(v.z), bf16x2_to_f16x2(v.w)) : v;
}
// The same for own keys and values, held as the cache would hold them: NaN counts as 0 and magnitudes saturate, because a token's
// row is multiplied by the zero probabilities of the tokens in front of it.
__device__ __forceinline__ uint4 as_held(uint4 v, bool bf16) {
  v = as_f16(v, bf16);
  return make_uint4(finite_f16x2(v.x), finite_f16x2(v.y), finite_f16x2(v.z), finite_f16x2(v.w));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

__device__ __forceinline__ void store_out(const Attn4Params& p, size_t at, float v) {
  if (p.out_bf16) reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
  else reinterpret_cast<__half*>(p.out)[at] = __float2half_rn(v);
}

__device__ __forceinline__ void store_out4(const Attn4Params& p, size_t at, float4 v) {
  *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.out) + at) =
      p.out_bf16 ? make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)) : make_uint2(pack_f16x2(v.x, v.y), pack_f16x2(v.z, v.w));
}
__device__ __forceinline__ void add_scaled(float4& a, float f, const float4& v) {
  a.x += f * v.x; a.y += f * v.y; a.z += f * v.z; a.w += f * v.w;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Another CTA's shared memory at the same place as this CTA's `addr`.
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, int cta) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}
__device__ __forceinline__ float2 load_peer2(uint32_t addr, int cta) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(peer_addr(addr, cta)) : "memory");
  return v;
}
__device__ __forceinline__ float4 load_peer4(uint32_t addr, int cta) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(peer_addr(addr, cta))
               : "memory");
  return v;
}

// CTAs that an SM holds at once (128 and 168 registers a thread).
__host__ __device__ constexpr int ctas_per_sm(int nt) { return nt == 1 ? 4 : 3; }

template <int HD, int NT>
struct Smem4 {
  static constexpr int kWarp = kStages * 2 * Kv4<HD>::kBlock;
  static constexpr int kStagesBytes = kWarps * kWarp;
  static constexpr int kPad = HD + 4;                                  // row stride of the partial results, in floats
  static constexpr int kPartBytes = kWarps * 8 * NT * kPad * 4;
  static constexpr int kStatBytes = kWarps * 8 * NT * 2 * 4;
  static constexpr int kJoinBytes = 8 * NT * (HD * 4 + 8);             // one CTA's results, for the others of its cluster
  static constexpr int kEnd = kPartBytes + kStatBytes + kJoinBytes;
  static constexpr int kUnion = kStagesBytes > kEnd ? kStagesBytes : kEnd;
  static_assert((kPartBytes + kStatBytes) % 16 == 0, "the joined rows are read in 16-byte pieces");
  // from 16 query rows on, the query operands do not fit the registers beside the accumulators
  static constexpr int kQBytes = NT > 1 ? 8 * NT * HD * 2 : 0;
  static constexpr int kScaleBytes = kWarps * 8 * NT * 4;
  static constexpr int kTotal = kUnion + kQBytes + kScaleBytes;
  static_assert(2 * Kv4<HD>::kBlock >= kPage * HD * 2, "a page of own values must fit in one stage");
};

// What each piece of a cut range weighs in the output of query row r: 2^(its reference - the largest) / the whole sum. One warp,
// two pieces a lane.
__device__ __forceinline__ void piece_weights(const Attn4Params& p, const AttnItem& it, int r, int lane, float* weight) {
  const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + static_cast<size_t>(it.slot0) * kAttn4Rows + r;
  float2 x[2];
  float M = kNoMax, sum = 0.f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int s = lane + 32 * j;
    x[j] = s < it.n_splits ? __ldcg(ml + s * kAttn4Rows) : make_float2(kNoMax, 0.f);
    M = fmaxf(M, x[j].x);
  }
  M = warp_max(M);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    x[j].x = fast_exp2(x[j].x - M);
    sum += x[j].x * x[j].y;
  }
  sum = warp_sum(sum);
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (lane + 32 * j < it.n_splits) weight[lane + 32 * j] = x[j].x * inv;
}

// NT = number of 8-row tiles of query rows (1 or 2).
template <int HD, int NT>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(NT))
attention_4bit_kernel(const Attn4Params p, const AttnItem* __restrict__ items) {
  using L = Kv4<HD>;
  using S = Smem4<HD, NT>;
  constexpr int NG = L::kGroups;            // channel groups
  constexpr int MT = HD / 16;               // 16-channel tiles of the output
  constexpr bool kQInRegs = S::kQBytes == 0;
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
  const int end_cached = min(it.tile_end, cached_pages);

  // A round is two pages: half a warp copies each.
  const int half = lane >> 4, sub = (lane & 15) * 16;
  const uint8_t* src0 = p.pool + static_cast<size_t>(it.kv_head) * L::kBlock + sub;
  const uint32_t dst0 = my_u + half * L::kBlock + sub;
  auto fetch = [&](int pg, int32_t id, int stage_off) {
    if (pg + half >= end_cached) return;
    if (!debug_in_range(id >= 0 && id < p.num_pages, p.status)) id = 0;
    const uint8_t* src = src0 + static_cast<size_t>(id) * page_stride;
    const uint32_t dst = dst0 + stage_off;
#pragma unroll
    for (int c = 0; c < L::kBlock / 256; ++c) cp_async_16(dst + c * 256, src + c * 256);
    if (L::kBlock % 256 && sub < L::kBlock % 256) cp_async_16(dst + L::kBlock / 256 * 256, src + L::kBlock / 256 * 256);
  };
  constexpr int kStep = 2 * kWarps;            // pages between a warp's rounds
  constexpr int kStageBytes = 2 * L::kBlock;
  const int pg0 = it.tile_begin + 2 * warp;
  auto page_id = [&](int pg) -> int32_t { return pg + half < end_cached ? __ldg(table + pg + half) : 0; };
  // No kernel writes the page table or the work list: they are read ahead of the wait. Where nothing that precedes this kernel on
  // the stream writes the cache either (the verification pass), the first pages are requested before it too; a caller who has just
  // appended waits first.
  int32_t ids[kStages];
#pragma unroll
  for (int st = 0; st < kStages; ++st) ids[st] = page_id(pg0 + st * kStep);
  if (!p.cache_is_settled) pdl_wait();
#pragma unroll
  for (int st = 0; st < kStages - 1; ++st) {
    fetch(pg0 + st * kStep, ids[st], st * kStageBytes);
    cp_async_commit();
  }
  int32_t id_ahead = ids[kStages - 1];
  if (p.cache_is_settled) pdl_wait();

  // Query operands. Lane (g, q) holds, for each group and each of the two words of a key row's chunk, the eight channels
  // 64 group + 16 q + 8 w .. + 7 of query row g of a tile: two k-steps of the score product.
  uint4 qr[kQInRegs ? NT : 1][NG][2];
  // operands of the product with a key's offsets and scales: sums of q over half a group each, -64 times the sums over the
  // channels held as 64 + c, high and low parts
  uint32_t qoff[NT], qscale[NT];
  // A row whose sums would leave fp16's range is taken times a power of two below 1, which the scale of its scores takes back:
  // channels that become subnormal by it lose 2^-25, where the row's largest is at least 2^14 / (64 x 16) = 16. The scales by row lie
  // in shared memory, a copy for each warp: registers for them are not left (two a tile: spills, 67.9 us for 66.7 on 64 contexts).
  float* row_scale = reinterpret_cast<float*>(smem + S::kUnion + S::kQBytes) + warp * 8 * NT;
  uint8_t* q_s = smem + S::kUnion;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = nt * 8 + g;
    uint4 v[NG][2];
    float sum[NG], sum64[NG], top = 0.f;
    const int t = (row0 + r) / G, hq = (row0 + r) % G;
#pragma unroll
    for (int grp = 0; grp < NG; ++grp) {
      sum[grp] = sum64[grp] = 0.f;
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
          if (i & 1) sum64[grp] += f.x + f.y;
        }
      }
      sum[grp] += __shfl_xor_sync(0xffffffffu, sum[grp], 1);     // lanes q = 0, 1 and q = 2, 3: half a group each
      sum64[grp] = -64.f * (sum64[grp] + __shfl_xor_sync(0xffffffffu, sum64[grp], 1));
      top = fmaxf(top, fmaxf(fabsf(sum[grp]), fabsf(sum64[grp])));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int down = max(0, static_cast<int>(__float_as_uint(top) >> 23) - 127 - 14);      // the sums end below 2^15
    if (__any_sync(0xffffffffu, down > 0)) {
      const float f = __uint_as_float(static_cast<uint32_t>(max(1, 127 - down)) << 23);
      const uint32_t f2 = pack_f16x2(f, f);
#pragma unroll
      for (int grp = 0; grp < NG; ++grp) {
        sum[grp] *= f;
        sum64[grp] *= f;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint4& x = v[grp][w];
          x = make_uint4(hmul2_u(x.x, f2), hmul2_u(x.y, f2), hmul2_u(x.z, f2), hmul2_u(x.w, f2));
        }
      }
    }
    if (q == 0) row_scale[r] = p.scale_log2e * __uint_as_float(static_cast<uint32_t>(127 + down) << 23);
#pragma unroll
    for (int grp = 0; grp < NG; ++grp)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if (kQInRegs) qr[nt][grp][w] = v[grp][w];
        else if (warp == 0) *reinterpret_cast<uint4*>(q_s + ((nt * NG + grp) * 2 + w) * 512 + lane * 16) = v[grp][w];
      }
    // A sum in two fp16 parts (22 bits): the lanes q of a row give a half group's high part, its low part, and the other half's.
    float part[2], part64[2];
#pragma unroll
    for (int grp = 0; grp < 2; ++grp) {
      const float f = grp < NG ? sum[grp < NG ? grp : 0] : 0.f, f64 = grp < NG ? sum64[grp < NG ? grp : 0] : 0.f;
      const float hi = __half2float(__float2half_rn(f)), hi64 = __half2float(__float2half_rn(f64));
      part[grp] = q & 1 ? f - hi : hi;
      part64[grp] = q & 1 ? f64 - hi64 : hi64;
    }
    qoff[nt] = pack_f16x2(part[0], part[1]);
    qscale[nt] = pack_f16x2(part64[0], part64[1]);
  }
  __syncwarp();
  if (!kQInRegs) __syncthreads();
  auto q_words = [&](int nt, int grp, int w) -> uint4 {
    if (kQInRegs) return qr[kQInRegs ? nt : 0][grp][w];
    return *reinterpret_cast<const uint4*>(q_s + ((nt * NG + grp) * 2 + w) * 512 + lane * 16);
  };

  float o[NT][MT][4];          // O^T without the offsets' share: channels 16 mt + g, + 8; query rows 2 q, 2 q + 1
  float oo[NT][4];             // sum_j p_j x_j of the quantity g mod 2 NG (offsets of the groups, then scales), and sum_j p_j
  float m_run[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m_run[nt][0] = m_run[nt][1] = kNoMax;
    oo[nt][0] = oo[nt][1] = oo[nt][2] = oo[nt][3] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
  }

  // Scores of NP x 16 keys (s[.][nt]: keys g, g + 8 x query rows 2 q, 2 q + 1) -> probabilities as operands of the output product.
  auto softmax = [&](auto np, auto& s, auto& pb) {
    constexpr int NP = decltype(np)::value;
    float2 scale[NT];            // of query rows 2 q, 2 q + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) scale[nt] = *reinterpret_cast<const float2*>(row_scale + nt * 8 + 2 * q);
    float top = kNoMax;
    float x[NP][NT][4];
#pragma unroll
    for (int pp = 0; pp < NP; ++pp)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[pp][nt][e] = fmaf(s[pp][nt][e], e & 1 ? scale[nt].y : scale[nt].x, -m_run[nt][e & 1]);
          top = fmaxf(top, x[pp][nt][e]);
        }
    if (__any_sync(0xffffffffu, top > kRaise)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float sc = e ? scale[nt].y : scale[nt].x;
          float mx = kNoMax;
#pragma unroll
          for (int pp = 0; pp < NP; ++pp) mx = fmaxf(mx, __fmul_rn(fmaxf(s[pp][nt][e], s[pp][nt][e + 2]), sc));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const float m_new = fmaxf(m_run[nt][e], mx - kHeadroom);
          const float corr = fast_exp2(m_run[nt][e] - m_new);
          m_run[nt][e] = m_new;
          oo[nt][e] *= corr;
          oo[nt][e + 2] *= corr;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            o[nt][mt][e] *= corr;
            o[nt][mt][e + 2] *= corr;
          }
#pragma unroll
          for (int pp = 0; pp < NP; ++pp) {
            // rounded as the maximum was: of scores above 2^24 the fused form would leave the products' roundings as exponents
            x[pp][nt][e] = __fsub_rn(__fmul_rn(s[pp][nt][e], sc), m_new);
            x[pp][nt][e + 2] = __fsub_rn(__fmul_rn(s[pp][nt][e + 2], sc), m_new);
          }
        }
    }
#pragma unroll
    for (int pp = 0; pp < NP; ++pp)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float (&y)[4] = x[pp][nt];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fast_exp2(y[e]);
        pb[pp][nt][0] = transpose8x8(pack_f16x2(y[0], y[1]));
        pb[pp][nt][1] = transpose8x8(pack_f16x2(y[2], y[3]));
      }
  };
  // Keys key0 .. key0 + 15 against the last key that the rows of token t see, base + per_token t: masked scores are -inf.
  auto mask = [&](float (&s)[NT][4], int key0, int base, int per_token) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = (row0 + nt * 8 + 2 * q + (e & 1)) / G;
        if (key0 + g + (e >> 1) * 8 > base + per_token * t) s[nt][e] = -INFINITY;
      }
  };

  const int see_base = it.ctx - (p.given ? 1 : 0), see_step = p.given ? 0 : 1;
  const int all_see = see_base + see_step * (row0 / G);        // the last key that every row of this tile sees
  auto cached_scores = [&](const uint8_t* b, float (&s)[NT][4]) {
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
        const uint32_t wa = kw[0][2 * grp + w], wb = kw[1][2 * grp + w], wa8 = wa >> 8, wb8 = wb >> 8;
        const uint32_t a0[4] = {codes_low(wa), codes_low(wb), codes64(wa), codes64(wb)};
        const uint32_t a1[4] = {codes_low(wa8), codes_low(wb8), codes64(wa8), codes64(wb8)};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 qv = q_words(nt, grp, w);
          if (w == 0) mma_k16_first(acc[nt][grp], a0, qv.x, qv.y);
          else mma_k16(acc[nt][grp], a0, qv.x, qv.y);
          mma_k16(acc[nt][grp], a1, qv.z, qv.w);
        }
      }
    // scales (fp32) and offsets of keys g and g + 8
    float sc[2][NG];
    uint32_t os[4];
    if (NG == 2) {
      const uint2 s2 = *reinterpret_cast<const uint2*>(b + L::kKScale + g * 8);
      const uint2 o2 = *reinterpret_cast<const uint2*>(b + L::kKOffset + g * 8);
      const float2 f0 = unpack_f16x2(s2.x), f1 = unpack_f16x2(s2.y);
      sc[0][0] = f0.x; sc[0][NG - 1] = f0.y; sc[1][0] = f1.x; sc[1][NG - 1] = f1.y;
      os[0] = o2.x; os[1] = o2.y; os[2] = s2.x; os[3] = s2.y;
    } else {
      const uint32_t s1 = *reinterpret_cast<const uint32_t*>(b + L::kKScale + g * 4);
      const float2 f = unpack_f16x2(s1);
      const uint32_t o1 = *reinterpret_cast<const uint32_t*>(b + L::kKOffset + g * 4);
      sc[0][0] = f.x; sc[1][0] = f.y;
      os[0] = __byte_perm(o1, o1, 0x1010); os[1] = __byte_perm(o1, o1, 0x3232);
      os[2] = __byte_perm(s1, s1, 0x1010); os[3] = __byte_perm(s1, s1, 0x3232);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mma_k16_first(s[nt], os, qoff[nt], qscale[nt]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int grp = 0; grp < NG; ++grp) s[nt][e] = fmaf(sc[e >> 1][grp], acc[nt][grp][e], s[nt][e]);
    }
  };

  // Value scales enter the products times 2^k, which the accumulators hold until the end: p s 2^k stays in fp16's normal range for
  // small values too. k is as large as the largest scale so far allows. (Costs 2 % at 8 query rows, 3 % at 16, and 1 % more for the
  // slots hidden below; a look at a share of the scales by each lane instead of all of them was no faster.)
  uint32_t v_up = k2Max, v_most = kMostAt2Max;             // 2^k; kKv4MaxScale 2^-k
  auto value_scales = [&](const uint8_t* b, uint32_t (&vs)[2 * NG]) {      // of keys 2 q, 2 q + 1 and 2 q + 8, 2 q + 9, by group
    if (NG == 2) *reinterpret_cast<uint4*>(vs) = *reinterpret_cast<const uint4*>(b + L::kVParams + q * 32 + 16);
    else *reinterpret_cast<uint2*>(vs) = *reinterpret_cast<const uint2*>(b + L::kVParams + q * 16 + 8);
  };
  auto scale_accumulators = [&](float f) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][mt][e] *= f;
  };
  // Slots of a warp's pages behind the last key that any row of the tile sees hold what the pages' last user left: their value
  // scales become zero, so that they have no say in k. (Their probabilities are zero.)
  const int last_seen = see_base + see_step * ((row0 + R - 1) / G);
  auto hide = [&](uint8_t* b, int pg) {
    if (pg * kPage + (lane & 15) + half * kPage > last_seen) {
      __half* at = reinterpret_cast<__half*>(b + half * L::kBlock + L::v_scale(lane & 15, 0));
      at[0] = __half(0.f);
      if (NG == 2) at[4] = __half(0.f);
    }
    __syncwarp();
  };
  auto fit_scales = [&](auto np, const uint8_t* b) {
    uint32_t top = v_most;
#pragma unroll
    for (int pp = 0; pp < decltype(np)::value; ++pp) {
      uint32_t vs[2 * NG];
      value_scales(b + pp * L::kBlock, vs);
#pragma unroll
      for (int i = 0; i < 2 * NG; ++i) top = hmax2_u(top, vs[i]);
    }
    if (!__any_sync(0xffffffffu, top != v_most)) return;
    const float2 f = unpack_f16x2(top);
    float most = fmaxf(f.x, f.y);
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    // the largest ends in [2^7, 2^8): a factor of 4 below where the next one has to give way
    const int k_was = static_cast<int>(v_up >> 26) - 15;
    const int k = max(0, min(k_was, 7 + 127 - static_cast<int>(__float_as_uint(most) >> 23)));
    v_up = (15 + k) * 0x04000400u;
    const float most_k = kKv4MaxScale * __uint_as_float((127 - k) << 23);
    v_most = pack_f16x2(most_k, most_k);
    scale_accumulators(__uint_as_float((127 + k - k_was) << 23));
  };
  auto cached_values = [&](const uint8_t* b, uint32_t (&pb)[NT][2]) {
    // (p s) (c - 8) by group
    uint32_t vs[2 * NG];
    value_scales(b, vs);
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) vs[i] = hmul2_u(vs[i], v_up);
    const uint8_t* vb = b + L::kVCodes + L::v_chunk(g, q) * 16;
#pragma unroll
    for (int grp = 0; grp < NG; ++grp) {
      uint32_t ps[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        ps[nt][0] = hmul2_u(pb[nt][0], vs[2 * grp]);
        ps[nt][1] = hmul2_u(pb[nt][1], vs[2 * grp + 1]);
      }
      const uint4 vw = *reinterpret_cast<const uint4*>(vb + grp * 512);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = word(vw, i), w8 = w >> 8;
        const uint32_t a[4] = {centred_low(w), centred_high(w), centred_low(w8), centred_high(w8)};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_k16(o[nt][4 * grp + i], a, ps[nt][0], ps[nt][1]);
      }
    }
    // offsets, scales and ones as the rows of one more product: sum_j p_j o_j, sum_j p_j s_j (which takes the 8 back at the end)
    // and sum_j p_j
    const uint2 vo = *reinterpret_cast<const uint2*>(b + L::kVParams + (q * 2 * NG + (g & (2 * NG - 1))) * 8);
    const uint32_t ao[4] = {vo.x, kOnes, vo.y, kOnes};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mma_k16(oo[nt], ao, pb[nt][0], pb[nt][1]);
  };

  // A page of the step's own keys and values, given as rows in fp16 or bf16: K operands straight from global memory, V through
  // this warp's last stage, which is not in use yet, and transposing loads.
  uint8_t* own_v = my + (kStages - 1) * kStageBytes;
  auto own_page = [&](int key0) {
    __syncwarp();
    constexpr int CH = HD / 8;
    for (int c = lane; c < kPage * CH; c += 32) {
      const int key = c / CH, ch = c % CH;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (key0 + key < it.n_new)
        v = as_held(*reinterpret_cast<const uint4*>(p.v_new + (it.tok0 + key0 + key) * p.kv_stride + it.kv_head * HD + ch * 8),
                   p.in_bf16 != 0);
      *reinterpret_cast<uint4*>(own_v + key * HD * 2 + ((ch ^ (key & 7)) << 4)) = v;
    }
    __syncwarp();
    float s1[1][NT][4];
    float (&s)[NT][4] = s1[0];
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
            x[j] = as_held(*reinterpret_cast<const uint4*>(p.k_new + (it.tok0 + key) * p.kv_stride + it.kv_head * HD + grp * 64 +
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
    uint32_t pb1[1][NT][2];
    softmax(std::integral_constant<int, 1>{}, s1, pb1);
    const uint32_t (&pb)[NT][2] = pb1[0];
    // matrices of an operand tile: channels 0-7 / 8-15 x keys 0-7, then x keys 8-15
    const int key = (lane & 7) + (lane >> 4) * 8, up = (lane >> 3) & 1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      uint32_t a[4];
      ldmatrix_x4_trans(a, smem_u32(own_v) + key * HD * 2 + (((2 * mt + up) ^ (key & 7)) << 4));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_k16(o[nt][mt], a, pb[nt][0], pb[nt][1]);
    }
    const uint32_t ao[4] = {0u, kOnes, 0u, kOnes};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mma_k16(oo[nt], ao, pb[nt][0], pb[nt][1]);
    __syncwarp();
  };

  // own pages first, while the cached ones are on their way, from the last warp on, which has the fewest of those
  for (int own = max(it.tile_begin, cached_pages) + (kWarps - 1 - warp); own < it.tile_end; own += kWarps)
    own_page((own - cached_pages) * kPage);

  if (it.tile_end > cached_pages) scale_accumulators(__uint_as_float((127 + kMaxUp) << 23));
  int stage_off = 0, ahead_off = (kStages - 1) * kStageBytes;
#pragma unroll 1
  for (int pg = pg0; pg < end_cached; pg += kStep) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    // the stage read in the previous round is free: request the round kStages - 1 ahead, and look up the one behind it
    fetch(pg + (kStages - 1) * kStep, id_ahead, ahead_off);
    cp_async_commit();
    id_ahead = page_id(pg + kStages * kStep);
    uint8_t* b = my + stage_off;
    if (pg + 1 < end_cached) {
      float s[2][NT][4];
      uint32_t pb[2][NT][2];
      cached_scores(b, s[0]);
      cached_scores(b + L::kBlock, s[1]);
      if (pg * kPage + 2 * kPage - 1 > all_see) {
        mask(s[0], pg * kPage, see_base, see_step);
        mask(s[1], pg * kPage + kPage, see_base, see_step);
        hide(b, pg);
      }
      softmax(std::integral_constant<int, 2>{}, s, pb);
      fit_scales(std::integral_constant<int, 2>{}, b);
      cached_values(b, pb[0]);
      cached_values(b + L::kBlock, pb[1]);
    } else {
      float s[1][NT][4];
      uint32_t pb[1][NT][2];
      cached_scores(b, s[0]);
      mask(s[0], pg * kPage, see_base, see_step);
      hide(b, pg);
      softmax(std::integral_constant<int, 1>{}, s, pb);
      fit_scales(std::integral_constant<int, 1>{}, b);
      cached_values(b, pb[0]);
    }
    ahead_off = stage_off;                       // the stage just read is the next to be filled
    stage_off = stage_off == (kStages - 1) * kStageBytes ? 0 : stage_off + kStageBytes;
  }
  cp_async_wait<0>();
  __syncthreads();

  // ------------------------------------------------------------------ the warps' results, joined in warp order
  float* po = reinterpret_cast<float*>(smem);                            // [warp][8 NT rows][HD + 4]
  float* pml = reinterpret_cast<float*>(smem + S::kPartBytes);           // [warp][8 NT rows][2]
  const float v_down = __uint_as_float((127 + 15 - (v_up >> 26)) << 23);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = nt * 8 + 2 * q + e;
      if (g == 0) {
        pml[(warp * 8 * NT + r) * 2] = m_run[nt][e];
        pml[(warp * 8 * NT + r) * 2 + 1] = oo[nt][e + 2];
      }
      float add[NG];             // what the offsets and the centring add to every channel of a group
#pragma unroll
      for (int grp = 0; grp < NG; ++grp)
        add[grp] = fmaf(8.f, __shfl_sync(0xffffffffu, oo[nt][e], (NG + grp) * 4 + q), __shfl_sync(0xffffffffu, oo[nt][e], grp * 4 + q));
      float* dst = po + (warp * 8 * NT + r) * S::kPad + g;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        dst[mt * 16] = fmaf(o[nt][mt][e], v_down, add[mt / 4]);
        dst[mt * 16 + 8] = fmaf(o[nt][mt][e + 2], v_down, add[mt / 4]);
      }
    }
  }
  __syncthreads();
  constexpr int kQuads = HD / 4;
  float4* joined = reinterpret_cast<float4*>(smem + S::kPartBytes + S::kStatBytes);      // cluster: [8 NT rows][HD / 4] of this CTA
  float2* joined_ml = reinterpret_cast<float2*>(joined + 8 * NT * kQuads);
  auto write_out = [&](int r, int c4, float4 v, float scale) {
    const int t = (row0 + r) / G, hq = (row0 + r) % G;
    store_out4(p, (it.tok0 + t) * p.out_stride + (it.kv_head * G + hq) * HD + 4 * c4,
               make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale));
  };
  for (int idx = threadIdx.x; idx < R * kQuads; idx += kThreads) {
    const int r = idx / kQuads, c4 = idx % kQuads;
    float M = kNoMax;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, pml[(w * 8 * NT + r) * 2]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = fast_exp2(pml[(w * 8 * NT + r) * 2] - M);
      add_scaled(acc, f, *reinterpret_cast<const float4*>(po + (w * 8 * NT + r) * S::kPad + 4 * c4));
      sum += f * pml[(w * 8 * NT + r) * 2 + 1];
    }
    if (p.cluster > 1) {
      joined[r * kQuads + c4] = acc;
      if (c4 == 0) joined_ml[r] = make_float2(M, sum);
    } else if (it.n_splits == 1) {
      write_out(r, c4, acc, sum > 0.f ? 1.f / sum : 0.f);
    } else {
      reinterpret_cast<float4*>(p.part_o)[(static_cast<size_t>(it.slot) * kAttn4Rows + r) * kQuads + c4] = acc;
      if (c4 == 0)
        reinterpret_cast<float2*>(p.part_ml)[static_cast<size_t>(it.slot) * kAttn4Rows + r] = make_float2(M, sum);
    }
  }
  if (p.cluster <= 1) return;

  // ------------------------------------------------------------------ the cluster's CTAs hold the pieces of one range
  cluster_barrier();
  const uint32_t rank = cluster_rank();
  const uint32_t joined_u = smem_u32(joined), ml_u = smem_u32(joined_ml);
  for (int idx = rank * kThreads + threadIdx.x; idx < R * kQuads; idx += kThreads * p.cluster) {
    const int r = idx / kQuads, c4 = idx % kQuads;
    float M = kNoMax;
    for (int c = 0; c < p.cluster; ++c) M = fmaxf(M, load_peer2(ml_u + r * 8, c).x);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int c = 0; c < p.cluster; ++c) {
      const float2 ml = load_peer2(ml_u + r * 8, c);
      const float f = fast_exp2(ml.x - M);
      add_scaled(acc, f, load_peer4(joined_u + (r * kQuads + c4) * 16, c));
      sum += f * ml.y;
    }
    write_out(r, c4, acc, sum > 0.f ? 1.f / sum : 0.f);
  }
  cluster_barrier();                 // nobody leaves while its results may still be read
}

// Pieces of one (step, kv head, row tile) -> output. One CTA per cut range and query row, one thread per channel: the pieces'
// weights once, in parallel, then a sum over the pieces in their order.
template <int HD>
__global__ void __launch_bounds__(HD) attention_4bit_merge_kernel(const Attn4Params p, const AttnItem* __restrict__ items, int tile) {
  __shared__ float weight[kAttn4MaxPieces];
  pdl_launch_dependents();
  const AttnItem it = items[blockIdx.x];
  const int G = p.n_q_heads / p.n_kv_heads;
  const int r = blockIdx.y, d = threadIdx.x, n = it.n_splits;
  pdl_wait();
  if (r >= min(tile, it.n_new * G - it.q_tok0)) return;
  // four channels a thread; the warps (HD = 64: half warps) take every fourth piece, and their sums are added in order. The first
  // pieces are requested before the weights are known.
  constexpr int kQuads = HD / 4, kAhead = 4;
  __shared__ float4 part[4][kQuads];
  const int share = d / kQuads, c4 = d % kQuads;
  const float4* o = reinterpret_cast<const float4*>(p.part_o + (static_cast<size_t>(it.slot0) * kAttn4Rows + r) * HD) + c4;
  float4 first[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (share + 4 * j < n) first[j] = __ldcg(o + static_cast<size_t>(share + 4 * j) * kAttn4Rows * kQuads);
  if (threadIdx.x < 32) piece_weights(p, it, r, d, weight);
  __syncthreads();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (share + 4 * j < n) add_scaled(acc, weight[share + 4 * j], first[j]);
#pragma unroll 8
  for (int s = share + 4 * kAhead; s < n; s += 4)
    add_scaled(acc, weight[s], __ldcg(o + static_cast<size_t>(s) * kAttn4Rows * kQuads));
  part[share][c4] = acc;
  __syncthreads();
  const float* sums = reinterpret_cast<const float*>(part);
  const int t = (it.q_tok0 + r) / G, hq = (it.q_tok0 + r) % G;
  store_out(p, (it.tok0 + t) * p.out_stride + (it.kv_head * G + hq) * HD + d, sums[d] + sums[HD + d] + sums[2 * HD + d] + sums[3 * HD + d]);
}

template <int HD, int NT>
cudaError_t opt_in() {
  static std::atomic<uint64_t> smem_opted{0};
  return opt_in_dynamic_smem(attention_4bit_kernel<HD, NT>, Smem4<HD, NT>::kTotal, smem_opted);
}

template <int HD, int NT>
cudaError_t launch_4bit(const Attn4Params& p, const AttnItem* items, int n_items, int n_merge, cudaStream_t s) {
  if (cudaError_t e = opt_in<HD, NT>(); e != cudaSuccess) return e;
  cudaError_t e = p.cluster > 1 ? launch_pdl_cluster(attention_4bit_kernel<HD, NT>, dim3(n_items), dim3(kThreads),
                                                     Smem4<HD, NT>::kTotal, s, p.cluster, p, items)
                                : launch_pdl(attention_4bit_kernel<HD, NT>, dim3(n_items), dim3(kThreads), Smem4<HD, NT>::kTotal, s,
                                             p, items);
  count_launch();
  if (e != cudaSuccess || n_merge == 0) return e != cudaSuccess ? e : cudaGetLastError();
  e = launch_pdl(attention_4bit_merge_kernel<HD>, dim3(n_merge, 8 * NT), dim3(HD), 0, s, p, items + n_items, 8 * NT);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// 8 or 16 query rows per work item; longer steps are cut into tiles of 16, whose items run side by side and find one another's
// pages in L2. (Tiles of 32 rows need 255 registers and two CTAs per SM: 28 rows over 83 K keys x 4 heads took 99 us, as two
// tiles of 16 45 us.)
int attention_4bit_row_tile(int max_rows) { return max_rows <= 8 ? 8 : 16; }

cudaError_t prepare_attention_4bit(int head_dim) {
  cudaError_t e = head_dim == 128 ? opt_in<128, 1>() : opt_in<64, 1>();
  if (e == cudaSuccess) e = head_dim == 128 ? opt_in<128, 2>() : opt_in<64, 2>();
  return e;
}

int attention_4bit_ctas_per_sm(int row_tile) { return ctas_per_sm(row_tile / 8); }

cudaError_t launch_attention_4bit(const Attn4Params& p, const AttnItem* items, int n_items, int n_merge, int row_tile,
                                  cudaStream_t s) {
  if (n_items <= 0) return cudaSuccess;
  if (p.head_dim == 128)
    return row_tile == 8 ? launch_4bit<128, 1>(p, items, n_items, n_merge, s) : launch_4bit<128, 2>(p, items, n_items, n_merge, s);
  if (p.head_dim == 64)
    return row_tile == 8 ? launch_4bit<64, 1>(p, items, n_items, n_merge, s) : launch_4bit<64, 2>(p, items, n_items, n_merge, s);
  return cudaErrorInvalidValue;
}

}  // namespace cs
