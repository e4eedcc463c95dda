// Products of 8-bit codes: out[t, n] = a_scale[t] w_scale[n] sum_k a[t, k] w[n, k], the sum in 32-bit integers on the tensor cores
// (tcgen05, kind::i8) and exact, whatever its order.
//
// Three forms by the number of tokens; a token has the same bits in all of them.
//   a few       vector: integer dot products of the ordinary cores, weights straight from global memory into registers
//   up to 128   narrow: the weights are the 128-row side of the product and the tokens its columns, so that a few tokens cost a few
//               columns; a CTA owns 128 output channels, all tokens and a piece of the k range, and the pieces of a tile are the
//               CTAs of a cluster, each of which collects the others' sums for its share of the tokens through distributed shared
//               memory
//   more        wide: pairs of CTAs over 256 tokens x 256 (or 128) rows of weights (below)
// Nothing is kept between calls and no global memory is used in between.
#include "i8.h"

#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace cs {

namespace {

constexpr int kBK = 128;                    // codes (= bytes) of a k block: one 128-byte swizzled row
constexpr int kTileBytes = 128 * kBK;       // 128 rows of it
constexpr int kMaxSplit = 8;                // CTAs along k of the narrow form: the largest cluster

// Map over rows of `bytes`-byte values, `stride` values apart: boxes whose rows are 64 or 128 bytes, swizzled alike. deep > 1: boxes of
// so many such pieces of every row, one after the other; `cols` is then a multiple of box_cols.
bool make_map(CUtensorMap* tm, void* base, CUtensorMapDataType type, int bytes, int64_t rows, int64_t cols, int64_t stride, int box_rows,
              int box_cols, int deep = 1) {
  using Encode = decltype(&cuTensorMapEncodeTiled);
  static const Encode encode = []() -> Encode {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                   q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<Encode>(p)
               : nullptr;
  }();
  if (!encode) return false;
  const int rank = deep > 1 ? 3 : 2;
  const auto u64 = [](int64_t v) { return static_cast<cuuint64_t>(v); };
  const cuuint64_t dims[3] = {u64(rank == 3 ? box_cols : cols), u64(rows), u64(cols / box_cols)};
  const cuuint64_t strides[2] = {u64(stride * bytes), u64(box_cols * bytes)};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), static_cast<cuuint32_t>(deep)};
  const cuuint32_t ones[3] = {1, 1, 1};
  return encode(tm, type, rank, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                box_cols * bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Time-outs of launches that are given no status word.
static __device__ uint32_t g_status;

// Instruction descriptor: signed 8-bit x signed 8-bit -> 32-bit integers, both operands K-major, tile M x N.
__host__ __device__ constexpr uint32_t idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
// D (+)= A B^T over one k block: four steps of 32 codes, the descriptors advancing by 32 bytes.
__device__ __forceinline__ void umma_i8_block(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred P;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "setp.ne.b32 P, %4, 0;\n\t"
      "add.u64 a1, %1, 2;\n\tadd.u64 b1, %2, 2;\n\t"
      "add.u64 a2, %1, 4;\n\tadd.u64 b2, %2, 4;\n\t"
      "add.u64 a3, %1, 6;\n\tadd.u64 b3, %2, 6;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, P;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], a1, b1, %3, 1;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], a2, b2, %3, 1;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], a3, b3, %3, 1;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void cluster_arrive_wait() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Where only the order of the CTAs' progress matters: a releasing arrival would wait for this thread's stores to global memory.
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t cta) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}
__device__ __forceinline__ void st_peer_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A sum with its scales, and what becomes of it. Every operation is rounded by itself, so that no form of the product fuses two of
// them and a token has the same bits in every batch.
__device__ __forceinline__ float scaled(uint32_t acc, float as, float ws) {
  return __fmul_rn(__fmul_rn(static_cast<float>(static_cast<int>(acc)), as), ws);
}
// The same without the conversion unit, which the exponential and the reciprocal of a gated tile keep busy: the upper half of the sum
// (its sign turned) and the lower half are put under the exponent of 2^23; the upper one times 2^16 less both offsets is exact, and
// adding the lower one rounds once.
__device__ __forceinline__ float scaled_by_parts(uint32_t acc, float as, float ws) {
  const float hi = __uint_as_float(__byte_perm(acc ^ 0x80000000u, 0x4b000000u, 0x7632));
  const float lo = __uint_as_float(__byte_perm(acc, 0x4b000000u, 0x7610));
  const float sum = __fadd_rn(fmaf(hi, 65536.0f, -(8388608.0f + 32768.0f) * 65536.0f - 8388608.0f), lo);
  return __fmul_rn(__fmul_rn(sum, as), ws);
}
// silu(y) y2, silu(y) = y / (1 + e^-y). The divisor is at least 1; beyond 2^126 its reciprocal is 0, which is what it tends to.
__device__ __forceinline__ float gate(float y, float y2) {
  const float d = __fadd_rn(1.0f, fast_exp2(__fmul_rn(y, -1.44269504f)));
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  return __fmul_rn(__fmul_rn(y, r), y2);
}

__device__ __forceinline__ void store_one(void* out, int64_t at, float v, int type) {
  if (type == kF16) static_cast<__half*>(out)[at] = __float2half_rn(v);
  else if (type == kBF16) static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(v);
  else static_cast<float*>(out)[at] = v;
}

// Clusters of c CTAs, one to an SM, that run at once: what cudaOccupancyMaxActiveClusters says on a B200, whose 148 SMs are not evenly
// spread over the groups that a cluster has to fit in.
constexpr int kClusters[9] = {0, 148, 74, 45, 33, 26, 22, 15, 15};

// -------------------------------------------------------------------------------------------------------- vector form
constexpr int kVectorTokens = 8;            // at most
constexpr int kVectorRows = 8;

__device__ __forceinline__ uint4 load_once(const int8_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ int dot16(uint4 a, uint4 b, int s) {
  s = __dp4a(static_cast<int>(a.x), static_cast<int>(b.x), s);
  s = __dp4a(static_cast<int>(a.y), static_cast<int>(b.y), s);
  s = __dp4a(static_cast<int>(a.z), static_cast<int>(b.z), s);
  return __dp4a(static_cast<int>(a.w), static_cast<int>(b.w), s);
}

// A CTA holds eight rows of weights (gated: four of each matrix), its warps and lanes 16 codes of k at a time. Bound by reading the
// weights: 1 x 1536 x 8960 4.7 us, 2.9 TB/s; smaller ones by latency (1 x 2048 x 1536 2.0 us), which is why all eight rows' loads leave
// before the first is used and before the tokens are waited for.
template <int TOKENS, bool GATED, int WARPS>
__global__ void __launch_bounds__(32 * WARPS)
gemm_i8_vector_kernel(const int8_t* a, int64_t a_stride, const int8_t* w, const int8_t* w2, const GemmI8 p) {
  constexpr int kChannels = GATED ? kVectorRows / 2 : kVectorRows;
  __shared__ int sums[WARPS][kVectorRows * TOKENS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n0 = blockIdx.x * kChannels;
  pdl_launch_dependents();
  if (!p.weights_settled) pdl_wait();
  const int8_t* row[kVectorRows];
#pragma unroll
  for (int r = 0; r < kVectorRows; ++r)      // rows past the last are the last once more
    row[r] = (GATED && r >= kChannels ? w2 : w) + static_cast<int64_t>(min(n0 + (GATED ? r % kChannels : r), p.N - 1)) * p.K;
  int s[kVectorRows][TOKENS] = {};
  bool waited = !p.weights_settled;
#pragma unroll 1
  for (int k = threadIdx.x * 16; k < p.K; k += WARPS * 512) {
    uint4 x[kVectorRows];
#pragma unroll
    for (int r = 0; r < kVectorRows; ++r) x[r] = load_once(row[r] + k);
    if (!waited) {
      pdl_wait();
      waited = true;
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      const uint4 y = *reinterpret_cast<const uint4*>(a + min(t, p.M - 1) * a_stride + k);
#pragma unroll
      for (int r = 0; r < kVectorRows; ++r) s[r][t] = dot16(x[r], y, s[r][t]);
    }
  }
  if (!waited) pdl_wait();
#pragma unroll
  for (int r = 0; r < kVectorRows; ++r)
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      const int sum = __reduce_add_sync(0xffffffffu, s[r][t]);
      if (lane == (r * TOKENS + t) % 32) sums[warp][r * TOKENS + t] = sum;
    }
  __syncthreads();
  const int c = threadIdx.x % kChannels, t = threadIdx.x / kChannels, n = n0 + c;
  if (t >= min(TOKENS, p.M) || n >= p.N) return;
  int sum = 0, sum2 = 0;
#pragma unroll
  for (int q = 0; q < WARPS; ++q) {
    sum += sums[q][c * TOKENS + t];
    if (GATED) sum2 += sums[q][(c + kChannels) * TOKENS + t];
  }
  const float as = p.a_scales[t];
  float v = scaled(static_cast<uint32_t>(sum), as, p.w_scales[n]);
  if (GATED) v = gate(v, scaled(static_cast<uint32_t>(sum2), as, p.w2_scales[n]));
  if (p.add) v = __fadd_rn(p.add[t * p.add_stride + n], v);
  store_one(p.out, t * p.out_stride + n, v, p.type);
}

template <bool GATED, int WARPS>
cudaError_t launch_vector(const GemmI8& p, int blocks, cudaStream_t s) {
  const auto kernel = p.M == 1   ? gemm_i8_vector_kernel<1, GATED, WARPS>
                      : p.M == 2 ? gemm_i8_vector_kernel<2, GATED, WARPS>
                      : p.M <= 4 ? gemm_i8_vector_kernel<4, GATED, WARPS>
                                 : gemm_i8_vector_kernel<8, GATED, 4>;
  const cudaError_t e = launch_pdl(kernel, dim3(blocks), dim3(32 * WARPS), 0, s, p.a, p.a_stride, p.w, p.w2, p);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}
template <bool GATED>
cudaError_t launch_vector(const GemmI8& p, cudaStream_t s) {
  const int channels = GATED ? kVectorRows / 2 : kVectorRows, blocks = (p.N + channels - 1) / channels;
  return blocks <= 2 * kNumSMs && p.M <= 4 ? launch_vector<GATED, 8>(p, blocks, s) : launch_vector<GATED, 4>(p, blocks, s);
}

// -------------------------------------------------------------------------------------------------------- narrow form
// Bound by reading the weights too: gated 8 x 18944 x 3584 25.0 us, 5.4 TB/s; 16 x 3584 x 18944 onto the residual 15.7 us, 4.4 TB/s (28
// tiles in clusters of four are 112 CTAs, and clusters of five are too many for the GPU). With 64 tokens and more the products' ends
// count: 64 x 1536 x 8960 8.5 us.
constexpr int kNarrowTokens = 128;
constexpr int kNarrowThreads = 320;         // warp 0: copies, warp 1: products, warps 2-9: results

template <int BN, bool GATED>
struct Narrow {
  static constexpr int kWTiles = GATED ? 2 : 1;
  // A stage is two k blocks (see the wide form): of the weights' 128 rows, of the second weights', and of the tokens.
  static constexpr int kTokenBlock = BN * kBK;
  static constexpr int kTokenOff = kWTiles * 2 * kTileBytes;
  static constexpr int kStageBytes = kTokenOff + 2 * kTokenBlock;
  static constexpr uint32_t kCols = kWTiles * BN < 32 ? 32 : kWTiles * BN;
  static constexpr int kBarOff = BN * 4;                    // behind the tokens' scales
  static constexpr int kHead = 1024;                        // scales and barriers, then the stages
  static constexpr int kMostStages = std::min(8, (224 * 1024 - kHead) / kStageBytes);
  // Shared memory of a CTA with so many stages, with slack for the tiles' alignment. CTAs that share an SM must find their columns
  // whenever they fit its shared memory: one that waited for columns while the rest of its cluster waited for it could wait for a CTA
  // that waits likewise.
  static constexpr int bytes(int stages) { return std::max(kHead + stages * kStageBytes + 1024, static_cast<int>(kCols) * 227 * 2 + 512); }
  static_assert(kMostStages >= 2 && bytes(kMostStages) <= 227 * 1024 && kBarOff + (2 * kMostStages + 2) * 8 <= kHead, "stages");
};

template <int BN, bool GATED>
__global__ void __launch_bounds__(kNarrowThreads)
gemm_i8_narrow_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w,
                      const __grid_constant__ CUtensorMap tm_w2, const GemmI8 p, int split, int log_own,
                      int stages, int deep) {
  using L = Narrow<BN, GATED>;
  constexpr uint32_t kIdesc = idesc_i8(128, BN);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* a_scales = reinterpret_cast<float*>(smem);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + L::kBarOff);
  uint64_t* empty_bar = full_bar + L::kMostStages;
  uint64_t* acc_bar = full_bar + 2 * L::kMostStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_bar + 1);
  smem += L::kHead;
  volatile uint32_t* abort_flag = tmem_slot + 1;
  uint32_t* status = p.status ? p.status : &g_status;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int piece = blockIdx.x % split, n0 = blockIdx.x / split * 128;
  const int kblocks = (p.K + kBK - 1) / kBK, kpairs = (kblocks + 1) / 2;
  const int kp0 = static_cast<int>(static_cast<int64_t>(kpairs) * piece / split);
  const int kp1 = static_cast<int>(static_cast<int64_t>(kpairs) * (piece + 1) / split);

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    mbar_init(acc_bar, 1);
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(&tm_w);
    if (GATED) tma_prefetch_desc(&tm_w2);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, L::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_launch_dependents();
  const auto load = [&](uint8_t* dst, const CUtensorMap* m, uint64_t* bar, int kp, int row, int block) {
    if (deep) {
      tma_load_3d(dst, m, bar, 0, row, 2 * kp);
    } else {
      tma_load_2d(dst, m, bar, 2 * kp * kBK, row);
      tma_load_2d(dst + block, m, bar, (2 * kp + 1) * kBK, row);      // zeros behind the last block
    }
  };
  const auto load_w = [&](int stage, int kp) {
    uint8_t* dst = smem + stage * L::kStageBytes;
    mbar_arrive_expect_tx(&full_bar[stage], L::kStageBytes);
    load(dst, &tm_w, &full_bar[stage], kp, n0, kTileBytes);
    if (GATED) load(dst + 2 * kTileBytes, &tm_w2, &full_bar[stage], kp, n0, kTileBytes);
  };
  // Weights that nothing in front of this launch writes are sent for at once, the tokens' rows after the wait.
  int ahead = 0;
  if (threadIdx.x == 0 && p.weights_settled)
    for (; ahead < stages && kp0 + ahead < kp1; ++ahead) load_w(ahead, kp0 + ahead);
  pdl_wait();

  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      for (int kp = kp0; kp < kp1; ++kp) {
        if (kp - kp0 >= ahead) {
          if (!mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, status)) { ok = false; break; }
          load_w(stage, kp);
        }
        load(smem + stage * L::kStageBytes + L::kTokenOff, &tm_a, &full_bar[stage], kp, 0, L::kTokenBlock);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
      // after a time-out: let the copies in flight land before the CTA goes away
      if (!ok)
        for (int i = 0; i < 64; ++i) __nanosleep(10000);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      const uint64_t wdesc0 = umma_desc_k128(smem_u32(smem));
      for (int kp = kp0; kp < kp1; ++kp) {
        if (!mbar_wait(&full_bar[stage], phase, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        const uint64_t wd = wdesc0 + static_cast<uint64_t>(stage * (L::kStageBytes >> 4));
        for (int b = 0; b < 2 && 2 * kp + b < kblocks; ++b) {
          const uint64_t wb = wd + b * (kTileBytes >> 4), ab = wd + (L::kTokenOff + b * L::kTokenBlock >> 4);
          umma_i8_block(tmem_base, wb, ab, kIdesc, kp != kp0 || b);
          if (GATED) umma_i8_block(tmem_base + BN, wb + (2 * kTileBytes >> 4), ab, kIdesc, kp != kp0 || b);
        }
        umma_commit(&empty_bar[stage]);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
      if (ok) umma_commit(acc_bar);
    }
  }
  __syncwarp();

  // ------------------------------------------------------------------ results: a thread per output channel, two warps per 32 channels
  const int quad = warp & 3, side = (warp - 2) >> 2;      // the lanes of tensor memory that this warp may read; which chunks it takes
  const bool results = warp >= 2;
  const int row = quad * 32 + lane;
  const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
  const int own0 = piece << log_own;                      // the 2^log_own tokens that this CTA writes
  const int n = n0 + row;
  float ws = 0.f, ws2 = 0.f;
  if (results) {
    const int t = threadIdx.x - 64;
    if (t < BN) a_scales[t] = t < p.M ? p.a_scales[t] : 0.f;
    if (n < p.N) {
      ws = p.w_scales[n];
      if (GATED) ws2 = p.w2_scales[n];
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    ok = __all_sync(0xffffffffu, mbar_wait(acc_bar, 0, abort_flag, status));
    tc_fence_after();
  }
  if (split > 1) {
    // Everybody's products are done with the stages: they become [piece][four tokens][weight matrix][128 channels][4].
    cluster_meet();
    if (results) {
      const uint32_t mine = smem_u32(smem) + static_cast<uint32_t>((piece << log_own) * L::kWTiles * 512 + row * 16);
#pragma unroll 1
      for (int c = side * 16; c < BN && c < p.M; c += 32) {
#pragma unroll
        for (int w = 0; w < L::kWTiles; ++w) {
          uint32_t r[16];
          tmem_ld_16(t_row + w * BN + c, r);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const int to = (c + j) >> log_own;
            if (to == piece || c + j >= p.M) continue;
            const uint32_t at = peer_addr(mine, to) + static_cast<uint32_t>(((c + j - (to << log_own)) * L::kWTiles + 4 * w) * 512);
            st_peer_v4(at, r[j], r[j + 1], r[j + 2], r[j + 3]);
          }
        }
      }
    }
    cluster_arrive_wait();
  }
  if (results && ok) {
    const int own1 = min(own0 + (1 << log_own), p.M);
#pragma unroll 1
    for (int c = (own0 & ~15) + side * 16; c < own1; c += 32) {
      uint32_t r[16], r2[16];
      float x[16];
      if (!GATED && p.add) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int64_t t = c + j;
          x[j] = t >= own0 && t < own1 && n < p.N ? p.add[t * p.add_stride + n] : 0.f;
        }
      }
      tmem_ld_16(t_row + c, r);
      if (GATED) tmem_ld_16(t_row + BN + c, r2);
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        if (c + j < own0 || c + j >= own1) continue;
        uint32_t s[4] = {r[j], r[j + 1], r[j + 2], r[j + 3]}, s2[4] = {r2[j], r2[j + 1], r2[j + 2], r2[j + 3]};
        const uint4* from = reinterpret_cast<const uint4*>(smem) + (c + j - own0) / 4 * L::kWTiles * 128 + row;
#pragma unroll 1
        for (int q = 0; q < split; ++q, from += (L::kWTiles * 32) << log_own) {
          if (q == piece) continue;
          const uint4 v = from[0];
          s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
          if (GATED) {
            const uint4 v2 = from[128];
            s2[0] += v2.x; s2[1] += v2.y; s2[2] += v2.z; s2[3] += v2.w;
          }
        }
        const float4 as4 = *reinterpret_cast<const float4*>(a_scales + c + j);
        const float as[4] = {as4.x, as4.y, as4.z, as4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t t = c + j + e;
          if (t >= own1 || n >= p.N) continue;
          float v = scaled(s[e], as[e], ws);
          if (GATED) v = gate(v, scaled(s2[e], as[e], ws2));
          else if (p.add) v = __fadd_rn(x[j + e], v);
          store_one(p.out, t * p.out_stride + n, v, p.type);
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, L::kCols);
  }
}

template <int BN, bool GATED>
cudaError_t launch_narrow(const CUtensorMap& ta, const CUtensorMap& tw, const CUtensorMap& tw2, const GemmI8& p, cudaStream_t s) {
  using L = Narrow<BN, GATED>;
  static std::atomic<uint64_t> opted{0};
  if (cudaError_t e = opt_in_dynamic_smem(gemm_i8_narrow_kernel<BN, GATED>, L::bytes(L::kMostStages), opted); e != cudaSuccess) return e;
  // As many pieces as there are SMs for, each with a pair of k blocks; fewer than four tokens are not shared out.
  const int tiles = (p.N + 127) / 128, kpairs = ((p.K + kBK - 1) / kBK + 1) / 2;
  int split = std::max(1, std::min(std::min(kMaxSplit, kpairs), kNumSMs / tiles));
  int log_own = 2;
  const auto fits = [&] {      // the clusters on the GPU, and what a CTA is handed over in two stages
    for (log_own = 2; (split << log_own) < BN;) ++log_own;
    return tiles <= kClusters[split] && (split << log_own) * L::kWTiles * 512 <= 2 * L::kStageBytes;
  };
  while (!fits() && split > 1) --split;
  // One CTA to an SM has it all; where there are more CTAs than SMs, two share it if their columns are few.
  const int two = (112 * 1024 - L::kHead) / L::kStageBytes;
  const int stages = tiles * split > kNumSMs && two >= 2 ? two : L::kMostStages;
  const dim3 grid(static_cast<unsigned>(tiles * split));
  const int deep = p.K % kBK == 0;
  const cudaError_t e = split > 1 ? launch_pdl_cluster(gemm_i8_narrow_kernel<BN, GATED>, grid, dim3(kNarrowThreads), L::bytes(stages), s,
                                                       split, ta, tw, tw2, p, split, log_own, stages, deep)
                                  : launch_pdl(gemm_i8_narrow_kernel<BN, GATED>, grid, dim3(kNarrowThreads), L::bytes(stages), s, ta, tw,
                                               tw2, p, split, log_own, stages, deep);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <bool GATED>
cudaError_t launch_by_tokens(const CUtensorMap& ta, const CUtensorMap& tw, const CUtensorMap& tw2, const GemmI8& p, cudaStream_t s) {
  switch (gemm_i8_box(p.M, p.N, p.K, GATED).rows) {
    case 16: return launch_narrow<16, GATED>(ta, tw, tw2, p, s);
    case 32: return launch_narrow<32, GATED>(ta, tw, tw2, p, s);
    case 64: return launch_narrow<64, GATED>(ta, tw, tw2, p, s);
    default: return launch_narrow<128, GATED>(ta, tw, tw2, p, s);
  }
}

// ---------------------------------------------------------------------------------------------------------- wide form
// Two CTAs (a pair) share a tile of 256 tokens x 256 rows of weights (gated: 128 of each matrix): each holds 128 rows of either
// operand, the leader issues products that read both CTAs' shared memory (cta_group::2), and each keeps the sums of its own 128
// tokens in its tensor memory, in one of two accumulators. Per SM and k block 32 KB are fetched for 512 cycles of products, half of
// what two separate 128 x 256 tiles would fetch. Bound by the tensor cores where tiles are many: gated 5377 x 8960 x 1536 101 us, 2910
// Top/s, gated 2038 x 18944 x 3584 168-175 us, 3200 Top/s; by the last turn of tiles at 350 of them (gated 1163 x 8960 x 1536 26.6 us,
// 2400 Top/s); by the copies, the exchange of sums and the ends where they are few (1163 x 1536 x 8960 17.8 us, 1800 Top/s).
constexpr int kWideThreads = 320;                      // warp 0: copies, warp 1: products, warps 2-9: results
// BN: rows of weights in a tile, each CTA holding half of them.
template <int BN>
struct Wide {
  // Two k blocks of both operands. A box costs the copy engine about 190 cycles besides its bytes, at 92 a cycle, so that two blocks a
  // box (32 KB) take 535 cycles a block, which the products take as well, and boxes of one take 735 (8192^3 363 us against 415).
  static constexpr int kWBlock = BN / 2 * kBK;
  static constexpr int kTokenBytes = 2 * kTileBytes;
  static constexpr int kStageBytes = kTokenBytes + 2 * kWBlock;
  static constexpr int kStages = BN == 256 ? 3 : 4;
  static constexpr int kBoxOff = kStages * kStageBytes;               // [8 warps] 32 rows of 32 results on their way out
  static constexpr int kBoxBytes = 4096;
  static constexpr int kScaleOff = kBoxOff + 8 * kBoxBytes;           // [256] scales of the tile's weights
  static constexpr int kBarOff = kScaleOff + 256 * 4;
  static constexpr int kTotal = kBarOff + 256 + 1024;
  static_assert(kTotal <= 227 * 1024, "shared memory");
};

// The same as umma_i8_block over the pair.
__device__ __forceinline__ void umma_i8_pair_block(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred Q;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "setp.ne.b32 Q, %4, 0;\n\t"
      "add.u64 a1, %1, 2;\n\tadd.u64 b1, %2, 2;\n\t"
      "add.u64 a2, %1, 4;\n\tadd.u64 b2, %2, 4;\n\t"
      "add.u64 a3, %1, 6;\n\tadd.u64 b3, %2, 6;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, Q;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], a1, b1, %3, 1;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], a2, b2, %3, 1;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], a3, b3, %3, 1;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Whether the phase is complete, without waiting.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred P;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 P, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, P;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Arrives at this barrier of every CTA of the mask once the products issued so far are done.
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar, uint32_t ctas) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_u32(bar)), "h"(static_cast<uint16_t>(ctas))
               : "memory");
}
// A copy into this CTA's shared memory that counts at a barrier of the pair's leader.
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* m, uint32_t leader_bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(leader_bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const CUtensorMap* m, uint32_t leader_bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(leader_bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// An arrival at another CTA's barrier that orders tensor-memory reads only (between the tcgen05 fences on either side): a release at
// cluster scope would wait for this thread's stores to global memory, 2500 cycles in which the products wait for the accumulator.
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n\t"
               "tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
// 32 consecutive results of one token per lane.
template <bool GATED>
__device__ __forceinline__ void results_of(const uint32_t (&r)[32], const uint32_t (&r2)[32], float as, const float* ws, const float* ws2,
                                           float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float4 w = reinterpret_cast<const float4*>(ws)[j];
    const float wj[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * j + e] = scaled(r[4 * j + e], as, wj[e]);
    if (GATED) {
      const float4 w2 = reinterpret_cast<const float4*>(ws2)[j];
      const float w2j[4] = {w2.x, w2.y, w2.z, w2.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = gate(v[4 * j + e], scaled_by_parts(r2[4 * j + e], as, w2j[e]));
    }
  }
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, const void* src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];\n\t"
               "cp.async.bulk.commit_group;" ::"l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(src)), "r"(x), "r"(y)
               : "memory");
}
// Until at most N of this thread's stores still read their shared memory.
template <int N>
__device__ __forceinline__ void tma_store_wait() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
constexpr int kOutBoxes = 0, kOutPieces = 1, kOutValues = 2;
// A warp's 32 rows x 32 columns through its box in shared memory, so that rows are written in whole 64- or 128-byte pieces (from the
// lanes' registers every store would touch 32 rows). Stores are boxes of a tensor map, or, where the residual is added, 16-byte pieces,
// or, where rows of the output are not made of 16-byte pieces, words and single values. Boxes of 16-bit results alternate between two
// places.
__device__ __forceinline__ void fill_box(uint8_t* box, const float (&v)[32], int lane, int type) {
  if (type != kF32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = v[8 * j + 2 * e], hi = v[8 * j + 2 * e + 1];
        w[e] = type == kF16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
      }
      *reinterpret_cast<uint4*>(box + lane * 64 + ((j ^ (lane >> 1 & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<float4*>(box + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  }
}
// The residual's pieces that add_pieces adds: sent for ahead of the products' results.
__device__ __forceinline__ void load_pieces(const GemmI8& p, int t0, int n0, int lane, float4 (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t t = t0 + 4 * i + (lane >> 3);
    x[i] = t < p.M && n0 + 32 <= p.N ? *reinterpret_cast<const float4*>(p.add + t * p.add_stride + n0 + 4 * (lane & 7))
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
__device__ __forceinline__ void add_pieces(const GemmI8& p, const uint8_t* box, int t0, int n0, int lane, const float4 (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 4 * i + (lane >> 3);
    const int64_t t = t0 + row;
    const float4 y = *reinterpret_cast<const float4*>(box + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
    if (t < p.M)
      *reinterpret_cast<float4*>(static_cast<float*>(p.out) + t * p.out_stride + n0 + 4 * (lane & 7)) =
          make_float4(__fadd_rn(x[i].x, y.x), __fadd_rn(x[i].y, y.y), __fadd_rn(x[i].z, y.z), __fadd_rn(x[i].w, y.w));
  }
}
// `width`: 32, or 64 for two boxes of 16-bit results side by side: the fewer pieces a row is written in, the fewer of them share a
// sector of memory with their neighbours.
__device__ __forceinline__ void write_values(const GemmI8& p, const uint8_t* box, int t0, int n0, int lane, int width) {
  const int rows = min(32, p.M - t0), cols = min(width, p.N - n0);
  if (p.type == kF32) {
    // a value a lane, eight rows at a time
    for (int r = 0; r < rows; r += 8) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[j] = p.add && r + j < rows && lane < cols ? p.add[(t0 + r + j) * p.add_stride + n0 + lane] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = r + j;
        const float y = *reinterpret_cast<const float*>(box + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4);
        if (row < rows && lane < cols) static_cast<float*>(p.out)[(t0 + row) * p.out_stride + n0 + lane] = p.add ? __fadd_rn(x[j], y) : y;
      }
    }
    return;
  }
  // A row at a time, a word a lane: of values 2 l, 2 l + 1 where the row begins on a word, else of 2 l + 1, 2 l + 2, and the last lane
  // has the first and the last value.
  const auto value = [&](int row, int c) {
    return *reinterpret_cast<const uint16_t*>(box + (c >> 5) * 2048 + row * 64 + (((c >> 3 & 3) ^ (row >> 1 & 3)) << 4) + (c & 7) * 2);
  };
  // eight rows at a time, so that their way through shared memory and out overlaps
  uint16_t* o = static_cast<uint16_t*>(p.out) + static_cast<int64_t>(t0) * p.out_stride + n0;
  const int first = static_cast<int>(reinterpret_cast<uintptr_t>(o) >> 1 & 1), turns = static_cast<int>(p.out_stride & 1);
#pragma unroll 1
  for (int r = 0; r < rows; r += 8, o += 8 * p.out_stride) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = 2 * lane + (first ^ (turns & j));
      w[j] = value(r + j, c) | static_cast<uint32_t>(value(r + j, c + 1 & 63)) << 16;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int odd = first ^ (turns & j), c = 2 * lane + odd;
      uint16_t* at = o + j * p.out_stride + c;
      const bool row_ok = r + j < rows;
      if (row_ok && c + 1 < cols) *reinterpret_cast<uint32_t*>(at) = w[j];
      if (row_ok && c + 1 == cols) *at = static_cast<uint16_t>(w[j]);
      if (row_ok && odd && lane == 31) at[-63] = static_cast<uint16_t>(w[j] >> 16);
    }
  }
}

template <bool GATED, int BN>
__global__ void __launch_bounds__(kWideThreads, 1)
gemm_i8_wide_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w,
                    const __grid_constant__ CUtensorMap tm_w2, const __grid_constant__ CUtensorMap tm_out, const GemmI8 p, int t_tiles,
                    int tiles, int split, int out_way, int deep) {
  using L = Wide<BN>;
  constexpr uint32_t kIdesc = idesc_i8(256, BN);
  constexpr int kOut = GATED ? BN / 2 : BN;            // output columns of a tile
  static_assert(!GATED || BN == 256, "the second matrix's sums begin at column 128");
  constexpr int kUnits = kOut / 32;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* scales = reinterpret_cast<float*>(smem + L::kScaleOff);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBarOff);
  uint64_t* full_bar = bars;                           // the leader's: both CTAs' copies of a stage
  uint64_t* empty_bar = bars + L::kStages;             // each CTA's own
  uint64_t* acc_full = bars + 2 * L::kStages;          // [2], each CTA's own
  uint64_t* acc_empty = bars + 2 * L::kStages + 2;     // [2], the leader's: both CTAs' eight warps
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * L::kStages + 4);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  uint32_t* status = p.status ? p.status : &g_status;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const uint32_t half = rank & 1, leader = rank & ~1u, pair_mask = 3u << leader;
  const int piece = rank >> 1;
  // k ranges are counted in pairs of blocks
  const int kblocks = (p.K + kBK - 1) / kBK, kpairs = (kblocks + 1) / 2;
  const int kp0 = static_cast<int>(static_cast<int64_t>(kpairs) * piece / split);
  const int kp1 = static_cast<int>(static_cast<int64_t>(kpairs) * (piece + 1) / split);
  const int first = blockIdx.x / (2 * split), step = gridDim.x / (2 * split);

  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&acc_full[a], 1);
      mbar_init(&acc_empty[a], 16);
    }
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(GATED && half ? &tm_w2 : &tm_w);
  }
  if (warp == 1) tmem_alloc_pair(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  cluster_arrive_wait();                               // the pair's barriers are ready
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_launch_dependents();

  // Token tiles run fastest: tiles that are in work together share their weights, and every weight is read from DRAM about once.
  const auto token0 = [&](int tile) { return (tile % t_tiles) * 256 + static_cast<int>(half) * 128; };
  const auto column0 = [&](int tile) { return tile / t_tiles * kOut; };
  const auto load = [&](uint8_t* dst, const CUtensorMap* m, uint32_t bar, int kp, int row, int block) {
    if (deep) {
      tma_load_3d_pair(dst, m, bar, 0, row, 2 * kp);
    } else {
      tma_load_2d_pair(dst, m, bar, 2 * kp * kBK, row);
      tma_load_2d_pair(dst + block, m, bar, (2 * kp + 1) * kBK, row);      // zeros behind the last block
    }
  };
  const auto load_w = [&](int stage, uint32_t bar, int kp, int tile) {
    uint8_t* dst = smem + stage * L::kStageBytes + L::kTokenBytes;
    if (GATED) load(dst, half ? &tm_w2 : &tm_w, bar, kp, column0(tile), L::kWBlock);
    else load(dst, &tm_w, bar, kp, column0(tile) + static_cast<int>(half) * (BN / 2), L::kWBlock);
  };
  int ahead = 0;
  if (threadIdx.x == 0 && p.weights_settled && first < tiles) {
    for (; ahead < L::kStages && kp0 + ahead < kp1; ++ahead) {
      if (!half) mbar_arrive_expect_tx(&full_bar[ahead], 2 * L::kStageBytes);
      load_w(ahead, peer_addr(smem_u32(&full_bar[ahead]), leader), kp0 + ahead, first);
    }
  }
  pdl_wait();

  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      for (int tile = first; tile < tiles && ok; tile += step) {
        for (int kp = kp0; kp < kp1; ++kp, ++issued) {
          const uint32_t bar = peer_addr(smem_u32(&full_bar[stage]), leader);
          if (issued >= ahead) {
            if (!mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, status)) { ok = false; break; }
            if (!half) mbar_arrive_expect_tx(&full_bar[stage], 2 * L::kStageBytes);
            load_w(stage, bar, kp, tile);
          }
          load(smem + stage * L::kStageBytes, &tm_a, bar, kp, token0(tile), kTileBytes);
          if (++stage == L::kStages) { stage = 0; phase ^= 1u; }
        }
      }
      // after a time-out: let the copies in flight land before the CTA goes away
      if (!ok)
        for (int i = 0; i < 64; ++i) __nanosleep(10000);
    }
  } else if (warp == 1) {
    // the whole warp keeps step, one elected thread issues: what it hands to the tensor cores is then known to be uniform
    if (!half) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ready = false;
      const uint64_t adesc0 = umma_desc_k128(smem_u32(smem)), bdesc0 = umma_desc_k128(smem_u32(smem) + L::kTokenBytes);
      for (int tile = first; tile < tiles && ok; tile += step) {
        if (!mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        for (int kp = kp0; kp < kp1; ++kp) {
          if (!ready && !mbar_wait(&full_bar[stage], phase, abort_flag, status)) { ok = false; break; }
          tc_fence_after();
          const int next = stage + 1 == L::kStages ? 0 : stage + 1;
          const uint32_t next_phase = next == 0 ? phase ^ 1u : phase;
          const uint64_t off = static_cast<uint64_t>(stage * (L::kStageBytes >> 4));
          ready = mbar_test(&full_bar[next], next_phase);
          if (elect_one()) {
            umma_i8_pair_block(tmem_base + acc * 256, adesc0 + off, bdesc0 + off, kIdesc, kp != kp0);
            if (2 * kp + 1 < kblocks)
              umma_i8_pair_block(tmem_base + acc * 256, adesc0 + off + (kTileBytes >> 4), bdesc0 + off + (L::kWBlock >> 4), kIdesc, 1);
            umma_commit_pair(&empty_bar[stage], pair_mask);
          }
          __syncwarp();
          stage = next;
          phase = next_phase;
        }
        if (!ok) break;
        if (elect_one()) umma_commit_pair(&acc_full[acc], pair_mask);
        __syncwarp();
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
      }
    }
  }
  __syncwarp();

  // ------------------------------------------------------------------ results: a thread per token, two warps per 32 tokens
  if (warp >= 2 || split > 1) {
    const bool results = warp >= 2;
    const int quad = warp & 3, side = (warp - 2) >> 2;
    const int row = quad * 32 + lane;
    const int own = kUnits / split;                    // 32-column units that this pair writes: own * piece ..
    const int u0 = own * piece + side * (own / 2), u1 = u0 + own / 2;      // this warp's
    uint8_t* box = smem + L::kBoxOff + (results ? warp - 2 : 0) * L::kBoxBytes;
    int acc = 0, turn = 0;
    uint32_t acc_phase = 0;
    for (int tile = first; tile < tiles; tile += step) {
      const int t = token0(tile) + row, n0 = column0(tile);
      float as = 0.f;
      if (results) {
        asm volatile("bar.sync 1, 256;" ::: "memory");        // the last tile's scales have been read
        // column c of the tile is row c of w, or of w2 behind the first 128 of a gated tile
        const int c = threadIdx.x - 64;
        const int n = n0 + (GATED ? c & 127 : c);
        scales[c] = n < p.N ? (GATED && c >= 128 ? p.w2_scales[n] : p.w_scales[n]) : 0.f;
        if (t < p.M) as = p.a_scales[t];
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, status));
        tc_fence_after();
      }
      const uint32_t t_row = tmem_base + acc * 256 + (static_cast<uint32_t>(quad * 32) << 16);
      if (split > 1) {
        // Everybody's products are done with the stages: they become [piece][own unit][matrix][4-column group][128 tokens][4].
        cluster_meet();
        if (results) {
          constexpr int kUnitBytes = (GATED ? 2 : 1) * 128 * 128;
          for (int i = side; i < kUnits; i += 2) {
            const int u = (i + own * (piece + 1)) % kUnits;      // everybody begins with another receiver
            const int to = u / own;
            if (to == piece) continue;
            const uint32_t at = peer_addr(smem_u32(smem) + static_cast<uint32_t>((piece * own + u - to * own) * kUnitBytes + row * 16),
                                          static_cast<uint32_t>(2 * to) + half);
#pragma unroll
            for (int w = 0; w < (GATED ? 2 : 1); ++w) {
              uint32_t r[32];
              tmem_ld_32x32(t_row + w * 128 + u * 32, r);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j)
                st_peer_v4(at + w * 16384 + j * 2048, r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
            }
          }
        }
        cluster_arrive_wait();
      }
      if (results) {
        for (int u = u0; u < u1; ++u) {
          const int t0 = token0(tile) + quad * 32, n = n0 + u * 32;
          if (!ok || n >= p.N) break;
          uint32_t r[32], r2[32];
          float4 x[8];
          if (!GATED && out_way == kOutPieces) load_pieces(p, t0, n, lane, x);
          tmem_ld_32x32(t_row + u * 32, r);
          if (GATED) tmem_ld_32x32(t_row + 128 + u * 32, r2);
          tmem_ld_wait();
          for (int q = 0; q < split; ++q) {
            if (q == piece) continue;
            const uint8_t* from = smem + (q * own + u - own * piece) * (GATED ? 2 : 1) * 16384 + row * 16;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint4 v = *reinterpret_cast<const uint4*>(from + j * 2048);
              r[4 * j] += v.x; r[4 * j + 1] += v.y; r[4 * j + 2] += v.z; r[4 * j + 3] += v.w;
              if (GATED) {
                const uint4 v2 = *reinterpret_cast<const uint4*>(from + 16384 + j * 2048);
                r2[4 * j] += v2.x; r2[4 * j + 1] += v2.y; r2[4 * j + 2] += v2.z; r2[4 * j + 3] += v2.w;
              }
            }
          }
          float v[32];
          results_of<GATED>(r, r2, as, scales + u * 32, scales + 128 + u * 32, v);
          uint8_t* to = box + (p.type == kF32 ? 0 : turn * 2048);
          if (out_way == kOutBoxes && lane == 0) {      // the box that was here has left
            if (p.type == kF32) tma_store_wait<0>();
            else tma_store_wait<1>();
          }
          __syncwarp();
          fill_box(to, v, lane, p.type);
          if (out_way == kOutBoxes) fence_proxy_async();
          __syncwarp();
          if (out_way == kOutBoxes) {
            if (lane == 0 && t0 < p.M) tma_store_2d(&tm_out, to, n, t0);
            turn ^= 1;
          } else if (!GATED && out_way == kOutPieces && n + 32 <= p.N) {
            add_pieces(p, to, t0, n, lane, x);
          } else if (p.type == kF32) {
            write_values(p, to, t0, n, lane, 32);
          } else if (turn || u + 1 == u1 || n + 32 >= p.N) {
            write_values(p, box, t0, n - 32 * turn, lane, 32 * (turn + 1));
            turn = 0;
          } else {
            turn = 1;                                    // together with the next one
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_at(peer_addr(smem_u32(&acc_empty[acc]), leader));
      }
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    }
  }

  if (warp >= 2 && lane == 0) tma_store_wait<0>();
  tc_fence_before();
  __syncthreads();
  cluster_meet();                                      // nobody leaves while the pair may still use its memory
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

template <bool GATED, int BN>
cudaError_t launch_wide(const CUtensorMap& ta, const CUtensorMap& tw, const CUtensorMap& tw2, const GemmI8& p, cudaStream_t s) {
  static std::atomic<uint64_t> opted{0};
  if (cudaError_t e = opt_in_dynamic_smem(gemm_i8_wide_kernel<GATED, BN>, Wide<BN>::kTotal, opted); e != cudaSuccess) return e;
  constexpr int kPairs = kNumSMs / 2, kOut = GATED ? BN / 2 : BN;
  const int64_t t_tiles = (static_cast<int64_t>(p.M) + 255) / 256, n_tiles = (p.N + kOut - 1) / kOut, tiles = t_tiles * n_tiles;
  if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
  const int kblocks = (p.K + kBK - 1) / kBK;
  int split = 1;
  // Handing sums over takes about as long as the products of 8 k blocks (300 x 1536 x 1536, 12 blocks: 8.0 us whole and cut in two;
  // 421 x 2048 x 2048: 9.6 and 9.1; 300 x 1536 x 3584: 12.9, 10.8 and, in four, 10.4; 735 x 1536 x 8960: 24.6 and 17.7).
  // fp32 results, whose rows are long to write, gain from more CTAs earlier (1163 x 1536 x 1536 onto the residual: 15.4 and 12.6).
  const int worth = p.type == kF32 ? 8 : 14;
  while (BN == 256 && split < (GATED ? 2 : 4) && tiles <= kClusters[4 * split] && kblocks >= worth * split) split *= 2;
  const int clusters = split > 1 ? static_cast<int>(tiles) : static_cast<int>(std::min<int64_t>(tiles, kPairs));
  const int bytes = p.type == kF32 ? 4 : 2;
  const bool pieces = reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && p.out_stride * bytes % 16 == 0 &&
                      (!p.add || (reinterpret_cast<uintptr_t>(p.add) % 16 == 0 && p.add_stride % 4 == 0));
  const int out_way = !pieces ? kOutValues : p.add ? kOutPieces : kOutBoxes;
  CUtensorMap tm_out = ta;
  if (out_way == kOutBoxes && !make_map(&tm_out, p.out, bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16,
                                        bytes, p.M, p.N, p.out_stride, 32, 32))
    return cudaErrorInvalidValue;
  const cudaError_t e = launch_pdl_cluster(gemm_i8_wide_kernel<GATED, BN>, dim3(clusters * 2 * split), dim3(kWideThreads), Wide<BN>::kTotal, s,
                                           2 * split, ta, tw, tw2, tm_out, p, static_cast<int>(t_tiles), static_cast<int>(tiles), split,
                                           out_way, p.K % kBK == 0 ? 1 : 0);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

namespace {
enum class Form { kVector, kNarrow, kWide, kWideHalf };
// Which form, as measured (us; weights not in L2).
// Vector: its dot products bind it from about 2^26 on (4 tokens x 1536 x 8960 5.4 against 6.8 narrow, 8 tokens 8.2 and 6.9; gated
// 4 x 8960 x 1536 9.0 and 8.8, 8 x 18944 x 3584 40 and 25), except that one and two tokens never do.
// Wide with tiles of 128 rows of weights (half): where all of them still run at once and the sum is not long. Their copies take 460
// cycles a block for half of the products, but a tile's end takes half as long and no sums are handed over (1163 x 1536 x 1536 6.9
// against 8.4 of whole tiles, 421 x 2048 x 2048 7.4 and 9.1, 421 x 2048 x 6144 14.3 and 13.8 cut in two, 1163 x 1792 x 4608, whose whole
// tiles are too many to be cut, 12.4 and 15.4).
// Between 64 and 128 tokens: narrow, unless whole tiles occupy half of the pairs (gated 128 x 8960 x 1536 10.9 against 14.0 narrow) or
// halves have a short sum (128 x 2048 x 1536 6.2 and 8.6; 128 x 3584 x 3584 10.1 and 9.6).
Form form_of(int M, int N, int K, bool gated) {
  const int64_t weights = static_cast<int64_t>(N) * K * (gated ? 2 : 1);
  if (M <= 2 || (M <= kVectorTokens && weights * (M <= 4 ? 4 : 8) <= 1 << 26)) return Form::kVector;
  if (M <= 64) return Form::kNarrow;
  const auto tiles = [&](int columns) { return (static_cast<int64_t>(M) + 255) / 256 * ((static_cast<int64_t>(N) + columns - 1) / columns); };
  const bool halves = !gated && K % kBK == 0 && tiles(128) <= kNumSMs / 2;
  if (M <= kNarrowTokens && tiles(gated ? 128 : 256) <= kNumSMs / 4 && !(halves && K <= 20 * kBK)) return Form::kNarrow;
  return halves && (K < 44 * kBK || tiles(256) > kClusters[4]) ? Form::kWideHalf : Form::kWide;
}
}  // namespace

I8Box gemm_i8_box(int M, int N, int K, bool gated) {
  const Form f = form_of(M, N, K, gated);
  if (f == Form::kVector) return {0, 0, false};
  return {f != Form::kNarrow ? 128 : M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128, f == Form::kWideHalf ? 64 : 128, K % kBK == 0};
}

bool make_i8_map(CUtensorMap* tm, const int8_t* base, int rows, int k, int64_t stride, int box_rows, bool deep) {
  return make_map(tm, const_cast<int8_t*>(base), CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, rows, k, stride, box_rows, kBK, deep ? 2 : 1);
}

cudaError_t gemm_i8(const CUtensorMap& ta, const CUtensorMap& tw, const CUtensorMap& tw2, const GemmI8& p, cudaStream_t s) {
  if (p.M <= 0) return cudaSuccess;
  const bool gated = p.w2 != nullptr;
  switch (form_of(p.M, p.N, p.K, gated)) {
    case Form::kVector: return gated ? launch_vector<true>(p, s) : launch_vector<false>(p, s);
    case Form::kNarrow: return gated ? launch_by_tokens<true>(ta, tw, tw2, p, s) : launch_by_tokens<false>(ta, tw, tw, p, s);
    case Form::kWideHalf: return launch_wide<false, 128>(ta, tw, tw, p, s);
    default: return gated ? launch_wide<true, 256>(ta, tw, tw2, p, s) : launch_wide<false, 256>(ta, tw, tw, p, s);
  }
}

cudaError_t i8_status(uint32_t* bits, cudaStream_t s) {
  cudaError_t e = cudaMemcpyFromSymbolAsync(bits, g_status, sizeof(uint32_t), 0, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess || *bits == 0) return e;
  const uint32_t zero = 0;
  e = cudaMemcpyToSymbolAsync(g_status, &zero, sizeof(uint32_t), 0, cudaMemcpyHostToDevice, s);
  return e == cudaSuccess ? cudaStreamSynchronize(s) : e;
}

}  // namespace cs
