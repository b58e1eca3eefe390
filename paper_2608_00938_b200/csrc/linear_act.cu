// y = act(x_scale[m] w_scale[n] (x @ w^T) + bias) + residual on tcgen05 tensor cores, bf16 or e4m3 operands, bf16 or fp32
// output: grace_linear's products with the epilogue that decoders with biases, smooth activations or 8-bit weights need.
//
// A k-block is 128 bytes of a row of either type (64 bf16, 128 e4m3) and four MMAs (K = 16 / K = 32), so both types share
// tiles, swizzle, descriptors and the dispatch rule of linear_form.cuh; an e4m3 product has half the k-blocks.
// act_kernel: one 128 x BN tile per CTA or per cluster that shares its K range.  act_pair_kernel: persistent CTA pairs on
// 256 x 256 tiles, two accumulators in TMEM, the epilogue of one under the products of the other.
#include "common.cuh"
#include "linear_form.cuh"
#include "tc.cuh"

namespace grace {

struct ActParams {
  const float *x_scale, *w_scale, *bias;                   // NULL: 1, 1, 0
  const void* residual;                                    // y's type, or NULL
  void* y;
  int64_t ldr, ldy;
  int M, N, KB, act;                                       // KB: k-blocks (the last one filled up with zeros)
};

// All activations but ReLU in the form v times a factor of (0, 1).
__device__ __forceinline__ float act_of(float v, int act) {
  switch (act) {
    case GRACE_ACT_RELU: return fmaxf(v, 0.f);
    case GRACE_ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    case GRACE_ACT_GELU_TANH: {
      const float t = v * fmaf(0.0713548162726f, v * v, 1.59576912160573f);      // 2 sqrt(2/pi) (v + 0.044715 v^3)
      return __fdividef(v, 1.f + __expf(-t));
    }
    case GRACE_ACT_SILU: return __fdividef(v, 1.f + __expf(-v));
    default: return v;
  }
}

template <bool F8, bool PAIR>
__device__ __forceinline__ void act_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (PAIR) {
    if (F8) tc::mma_ss_pair_f8(d, a, b, idesc, accumulate); else tc::mma_ss_pair(d, a, b, idesc, accumulate);
  } else {
    if (F8) tc::mma_ss_f8(d, a, b, idesc, accumulate); else tc::mma_ss(d, a, b, idesc, accumulate);
  }
}
template <bool F8>
__host__ __device__ constexpr uint32_t act_idesc(int M, int N) { return F8 ? tc::idesc_e4m3(M, N) : tc::idesc_bf16(M, N, 0); }

// ---------------------------------------------------------------------------------------------
// One 128 x BN tile per CTA; SPLIT > 1: a cluster of SPLIT CTAs shares a tile's K range, and each finishes BN / SPLIT of its
// columns from the partial sums that the others send through distributed shared memory (added in rank order).
// ---------------------------------------------------------------------------------------------
template <int BN, int STAGES, int SPLIT>
struct ActCfg {
  static constexpr int kABytes = 128 * 128, kBBytes = BN * 128, kStageBytes = kABytes + kBBytes;
  static constexpr int kSlice = BN / SPLIT;
  static constexpr int kXBytes = (SPLIT - 1) * 128 * kSlice * 4;
  static constexpr int kColBytes = kSlice * 8;             // (w_scale, bias) of the slice's columns
  static constexpr int kTotal = STAGES * kStageBytes + kXBytes + kColBytes + 1024 /*alignment slack*/ + 256 /*barriers*/;
  static_assert(kSlice % 16 == 0 && kTotal <= 227 * 1024, "");
};
constexpr int kActThreads = 192;                           // four row warps, TMA producer, MMA issuer

template <bool F8, bool F32, int BN, int STAGES, int SPLIT>
__global__ void __launch_bounds__(kActThreads, 2)
act_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const ActParams p) {
  using S = ActCfg<BN, STAGES, SPLIT>;
  constexpr bool kTriggerLate = S::kTotal <= tc::kMostSmemBesideTmemAll;
  if (!kTriggerLate) pdl_trigger();
  constexpr int kSlice = S::kSlice, kBK = F8 ? 128 : 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float4* xbuf = reinterpret_cast<float4*>(tiles + STAGES * S::kStageBytes);             // [SPLIT - 1][kSlice / 4][128]
  float* col_s = reinterpret_cast<float*>(tiles + STAGES * S::kStageBytes + S::kXBytes); // [kSlice] scales, [kSlice] biases
  uint64_t* full = reinterpret_cast<uint64_t*>(tiles + STAGES * S::kStageBytes + S::kXBytes + S::kColBytes);
  uint64_t* empty = full + STAGES;
  uint64_t* accum_bar = empty + STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(accum_bar + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = SPLIT > 1 ? (int)(blockIdx.x % SPLIT) : 0;
  const int m0 = blockIdx.y * kGemmBM, n0 = (int)(blockIdx.x / SPLIT) * BN;
  const int kb0 = p.KB * rank / SPLIT, KB = p.KB * (rank + 1) / SPLIT - kb0;             // this CTA's k-blocks (>= 1)

  if (SPLIT > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // "this CTA has started"
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { tc::mbar_init(full + s, 1); tc::mbar_init(empty + s, 1); }
    tc::mbar_init(accum_bar, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 4) {
    if (lane == 0) { tc::tma_prefetch_desc(&map_x); tc::tma_prefetch_desc(&map_w); }
    __syncwarp();
    tc::tmem_alloc(tmem_slot, BN < 32 ? 32 : BN);
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (kTriggerLate) pdl_trigger();                         // see tc::kMostSmemBesideTmemAll
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();

  bool ok = true;
  const int row = warp * 32 + lane;                        // warps 0..3: TMEM lane = row of the tile
  const int m = m0 + row;
  const int slice0 = n0 + rank * kSlice;                   // first of the columns this CTA finishes

  if (warp == 4) {
    if (lane == 0) {
      for (int kb = 0; kb < KB; ++kb) {
        const int s = kb % STAGES;
        if (kb >= STAGES && !tc::mbar_wait(empty + s, ((kb / STAGES) & 1) ^ 1, abort_flag)) break;
        tc::mbar_expect_tx(full + s, S::kStageBytes);
        uint8_t* a = tiles + s * S::kStageBytes;
        tc::tma_load_2d(a + S::kABytes, &map_w, full + s, (kb0 + kb) * kBK, n0);
        tc::tma_load_2d(a, &map_x, full + s, (kb0 + kb) * kBK, m0);
      }
    }
    __syncwarp();
  } else if (warp == 5) {
    if (lane == 0) {
      constexpr uint32_t idesc = act_idesc<F8>(kGemmBM, BN);
      for (int kb = 0; kb < KB; ++kb) {
        const int s = kb % STAGES;
        if (!tc::mbar_wait(full + s, (kb / STAGES) & 1, abort_flag)) break;
        tc::tc_fence_after();
        const uint32_t a_addr = tc::smem_addr(tiles + s * S::kStageBytes);
        const uint64_t a_desc = tc::smem_desc_sw128(a_addr, 16, 1024);
        const uint64_t b_desc = tc::smem_desc_sw128(a_addr + S::kABytes, 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          act_mma<F8, false>(tmem_base, a_desc + (uint64_t)(2 * k), b_desc + (uint64_t)(2 * k), idesc, (kb | k) ? 1u : 0u);
        tc::mma_commit(empty + s);
      }
      tc::mma_commit(accum_bar);
    }
    __syncwarp();
  } else {
    for (int i = threadIdx.x; i < kSlice; i += 128) {
      const int n = min(slice0 + i, p.N - 1);
      col_s[i] = p.w_scale != nullptr ? __ldg(p.w_scale + n) : 1.f;
      col_s[kSlice + i] = p.bias != nullptr ? __ldg(p.bias + n) : 0.f;
    }
    ok = tc::mbar_wait(accum_bar, 0, abort_flag);
    ok = __all_sync(kFullMask, ok);
    tc::tc_fence_after();
    tc::named_bar_sync(1, 128);                            // the column vectors of all four warps
  }
  const uint32_t t_acc = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
  if (SPLIT > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (warp < 4 && ok) {
#pragma unroll 1
      for (int o = 1; o < SPLIT; ++o) {
        const int dst = (rank + o) % SPLIT;
        const int slot = rank < dst ? rank : rank - 1;     // this CTA's place among the owner's SPLIT - 1 sources
        const uint32_t remote = tc::cluster_addr_of(xbuf + slot * (kSlice / 4) * 128 + row, (uint32_t)dst);
#pragma unroll
        for (int c = 0; c < kSlice; c += 16) {
          uint32_t acc[16];
          tc::tmem_ld16(t_acc + (uint32_t)(dst * kSlice + c), acc);
          tc::tmem_ld_wait();
          if (m < p.M) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};"
                           ::"r"(remote + (uint32_t)((c / 4 + j) * 128 * 16)), "r"(acc[4 * j]), "r"(acc[4 * j + 1]),
                             "r"(acc[4 * j + 2]), "r"(acc[4 * j + 3]) : "memory");
          }
        }
      }
    }
    __syncwarp();
    tc::cluster_sync_all();
  }

  if (warp < 4 && ok) {
    constexpr int kSize = F32 ? 4 : 2;
    const float xs = p.x_scale != nullptr ? __ldg(p.x_scale + min(m, p.M - 1)) : 1.f;
    // 16 columns of a row in wide accesses where both rows' starts allow them
    const bool wide_y = ((reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)(p.ldy * kSize)) & 15) == 0;
    const bool wide_r = ((reinterpret_cast<uintptr_t>(p.residual) | (uintptr_t)(p.ldr * kSize)) & 15) == 0;
    char* const yrow = reinterpret_cast<char*>(p.y) + (int64_t)m * p.ldy * kSize;
    const char* const rrow = reinterpret_cast<const char*>(p.residual) + (int64_t)m * p.ldr * kSize;
#pragma unroll 1
    for (int c = 0; c < kSlice; c += 16) {
      uint32_t acc[16];
      tc::tmem_ld16(t_acc + (uint32_t)(rank * kSlice + c), acc);
      const int n = slice0 + c;
      const bool in = m < p.M && n < p.N, whole = n + 16 <= p.N;
      uint4 res[kSize];                                    // 16 elements
#pragma unroll
      for (int j = 0; j < kSize; ++j) {
        res[j] = make_uint4(0, 0, 0, 0);
        if (in && p.residual != nullptr && whole && wide_r)  // (not .nc: the residual may be y itself)
          res[j] = reinterpret_cast<const uint4*>(rrow + (int64_t)n * kSize)[j];
      }
      tc::tmem_ld_wait();
      if (!in) continue;
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = SPLIT == 1 ? __uint_as_float(acc[j]) : 0.f;
      if (SPLIT > 1) {
        // in rank order, whoever owns the columns
#pragma unroll
        for (int s = 0; s < SPLIT; ++s) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float4 t = make_float4(__uint_as_float(acc[4 * j]), __uint_as_float(acc[4 * j + 1]),
                                   __uint_as_float(acc[4 * j + 2]), __uint_as_float(acc[4 * j + 3]));
            if (s != rank) t = xbuf[((s < rank ? s : s - 1) * (kSlice / 4) + c / 4 + j) * 128 + row];
            v[4 * j] += t.x; v[4 * j + 1] += t.y; v[4 * j + 2] += t.z; v[4 * j + 3] += t.w;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        const float4 ws = *reinterpret_cast<const float4*>(col_s + c + j);
        const float4 bb = *reinterpret_cast<const float4*>(col_s + kSlice + c + j);
        v[j] = act_of(fmaf(v[j] * xs, ws.x, bb.x), p.act); v[j + 1] = act_of(fmaf(v[j + 1] * xs, ws.y, bb.y), p.act);
        v[j + 2] = act_of(fmaf(v[j + 2] * xs, ws.z, bb.z), p.act); v[j + 3] = act_of(fmaf(v[j + 3] * xs, ws.w, bb.w), p.act);
      }
      if (p.residual != nullptr) {
        if (whole && wide_r) {
#pragma unroll
          for (int j = 0; j < kSize; ++j) {
            const uint32_t w[4] = {res[j].x, res[j].y, res[j].z, res[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (F32) {
                v[4 * j + e] += __uint_as_float(w[e]);
              } else {
                v[(8 * j + 2 * e) & 15] += bf16_lo(w[e]);
                v[(8 * j + 2 * e + 1) & 15] += bf16_hi(w[e]);
              }
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (n + j < p.N)
              v[j] += F32 ? reinterpret_cast<const float*>(rrow)[n + j]
                          : __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(rrow)[n + j] << 16);
        }
      }
      uint4 o[kSize];
#pragma unroll
      for (int j = 0; j < kSize; ++j)
        o[j] = F32 ? make_uint4(__float_as_uint(v[(4 * j) & 15]), __float_as_uint(v[(4 * j + 1) & 15]), __float_as_uint(v[(4 * j + 2) & 15]), __float_as_uint(v[(4 * j + 3) & 15]))
                   : make_uint4(pack_bf16x2(v[(8 * j) & 15], v[(8 * j + 1) & 15]), pack_bf16x2(v[(8 * j + 2) & 15], v[(8 * j + 3) & 15]),
                                pack_bf16x2(v[(8 * j + 4) & 15], v[(8 * j + 5) & 15]), pack_bf16x2(v[(8 * j + 6) & 15], v[(8 * j + 7) & 15]));
      if (whole && wide_y) {
#pragma unroll
        for (int j = 0; j < kSize; ++j) reinterpret_cast<uint4*>(yrow + (int64_t)n * kSize)[j] = o[j];
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (n + j < p.N) {
            if (F32) reinterpret_cast<float*>(yrow)[n + j] = v[j];
            else reinterpret_cast<__nv_bfloat16*>(yrow)[n + j] = __float2bfloat16_rn(v[j]);
          }
        }
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 4) tc::tmem_dealloc(tmem_base, BN < 32 ? 32 : BN);
}

// ---------------------------------------------------------------------------------------------
// Persistent CTA pairs: 256 x 256 tiles (n fastest), each CTA with 128 rows of x and 128 of the tile's rows of w in a ring of
// five stages, one tcgen05.mma stream per pair into one of two accumulators (all of TMEM).  Eight epilogue warps per CTA in
// two groups of four, each with 128 of the tile's columns and two staging buffers of 128 rows x 128 bytes: the residual comes
// into a buffer by TMA, the group adds it where it lies and hands the buffer to a TMA store, so that neither passes through
// strided accesses.  (Eight warps and not four: an e4m3 product of K = 512 has 2048 clocks of MMAs per tile, and a smooth
// activation takes an exponential and a quotient for each of 128 x 256 elements of a CTA.)
// ---------------------------------------------------------------------------------------------
constexpr int kAPStages = 5;
constexpr int kAPStageBytes = 2 * 128 * 128;
constexpr int kAPStaging = 128 * 128;
constexpr int kAPSmem = kAPStages * kAPStageBytes + 4 * kAPStaging + 256 + 2 * 256 * 4;
constexpr int kAPThreads = 320;
static_assert(kAPSmem >= tc::kTmemAllSmem && kAPSmem <= 227 * 1024, "");

template <bool F8, bool F32>
__global__ void __launch_bounds__(kAPThreads, 1)
act_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_r, const ActParams p) {
  extern __shared__ __align__(1024) uint8_t smem_pair[];
  uint8_t* tiles = smem_pair;
  if ((tc::smem_addr(tiles) & 1023u) != 0) {               // the swizzled tiles need it; same answer in every thread
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicAdd(&tc::g_tc_timeouts, 1);
    return;
  }
  uint8_t* staging = tiles + kAPStages * kAPStageBytes;    // [2 groups][2]
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + 4 * kAPStaging);       // even CTA only: both CTAs' bytes landed
  uint64_t* empty = full + kAPStages;                      // the pair's MMAs have read the stage
  uint64_t* acc_full = empty + kAPStages;                  // [2]
  uint64_t* acc_empty = acc_full + 2;                      // [2] even CTA only: 8 local + 8 remote epilogue warps
  uint64_t* res_full = acc_empty + 2;                      // [2 groups][2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(res_full + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* col_s = reinterpret_cast<float*>(staging + 4 * kAPStaging + 256);      // [256] scales, [256] biases

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_cta_rank();            // 0: issues the MMAs; 1: peer
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int n_tiles = (p.N + 255) / 256, total = n_tiles * ((p.M + 255) / 256);
  constexpr int kBK = F8 ? 128 : 64;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kAPStages; ++s) { tc::mbar_init(full + s, 1); tc::mbar_init(empty + s, 1); }
    for (int a = 0; a < 2; ++a) { tc::mbar_init(acc_full + a, 1); tc::mbar_init(acc_empty + a, 16); }
    for (int a = 0; a < 4; ++a) tc::mbar_init(res_full + a, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
    tc::tma_prefetch_desc(&map_x); tc::tma_prefetch_desc(&map_w); tc::tma_prefetch_desc(&map_y);
  }
  if (warp == 0) tc::tmem_alloc_pair(tmem_slot, 512);
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync_all();                                  // both CTAs' barriers exist before any remote arrive
  tc::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();                                              // everything above overlapped the previous kernel's tail
  pdl_trigger();

  if (warp == 0) {
    if (lane == 0) {                                        // ---- TMA producer (both CTAs) ----
      int it = 0;
      for (int tile = pair; tile < total; tile += n_pairs) {
        const int m0 = (tile / n_tiles) * 256 + (int)rank * 128, n0 = (tile % n_tiles) * 256 + (int)rank * 128;
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const int s = it % kAPStages;
          if (!tc::mbar_wait_cluster(empty + s, ((it / kAPStages) & 1) ^ 1, abort_flag)) { tile = total; break; }
          if (rank == 0) tc::mbar_expect_tx(full + s, 2 * kAPStageBytes);    // this CTA's bytes and the peer's
          uint8_t* a = tiles + s * kAPStageBytes;
          const uint32_t bar = tc::cluster_addr_of(full + s, 0);
          tc::tma_load_2d_pair(a, &map_x, bar, kb * kBK, m0);
          tc::tma_load_2d_pair(a + 128 * 128, &map_w, bar, kb * kBK, n0);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {                           // ---- even CTA: MMA issuer for the pair ----
      constexpr uint32_t idesc = act_idesc<F8>(256, 256);
      int it = 0, local = 0;
      for (int tile = pair; tile < total; tile += n_pairs, ++local) {
        const int ab = local & 1;
        if (!tc::mbar_wait_cluster(acc_empty + ab, ((local >> 1) & 1) ^ 1, abort_flag)) break;
        tc::tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(ab * 256);
        bool ok = true;
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const int s = it % kAPStages;
          if (!tc::mbar_wait_cluster(full + s, (it / kAPStages) & 1, abort_flag)) { ok = false; break; }
          tc::tc_fence_after();
          const uint32_t a_addr = tc::smem_addr(tiles + s * kAPStageBytes);
          const uint64_t a_desc = tc::smem_desc_sw128(a_addr, 16, 1024);
          const uint64_t b_desc = tc::smem_desc_sw128(a_addr + 128 * 128, 16, 1024);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            act_mma<F8, true>(d_tmem, a_desc + (uint64_t)(2 * k), b_desc + (uint64_t)(2 * k), idesc, (kb | k) ? 1u : 0u);
          tc::mma_commit_pair(empty + s, 3);
        }
        if (!ok) break;
        tc::mma_commit_pair(acc_full + ab, 3);
      }
    }
  } else {
    // ---- epilogue warps 2..9: group of 128 columns, TMEM lane quarter q = rows q*32 + lane of this CTA's 128 ----
    const int group = (warp - 2) >> 2, q = warp & 3, row = q * 32 + lane;
    const bool issuer = warp == 2 + 4 * group && lane == 0;
    constexpr int kCols = F32 ? 32 : 64, kChunks = 128 / kCols;                  // columns of a staging buffer
    uint8_t* const bufs = staging + group * 2 * kAPStaging;
    const bool res = p.residual != nullptr;
    int local = 0, g = 0;                                   // g: chunks of this group so far
    // chunk g's residual into its buffer; the stores that used the buffer have been read out of it (bulk_wait_read)
    auto fetch_residual = [&](int tile, int chunk, int at) {
      if (tile >= total) return;
      uint64_t* bar = res_full + 2 * group + (at & 1);
      tc::mbar_expect_tx(bar, kAPStaging);
      tc::tma_load_2d(bufs + (at & 1) * kAPStaging, &map_r, bar, (tile % n_tiles) * 256 + group * 128 + chunk * kCols,
                      (tile / n_tiles) * 256 + (int)rank * 128);
    };
    float xs_next = 1.f, ws_next = 1.f, bias_next = 0.f;
    auto fetch_vectors = [&](int tile) {                    // one tile ahead, from clamped addresses
      tile = min(tile, total - 1);
      const int m = min((tile / n_tiles) * 256 + (int)rank * 128 + row, p.M - 1), n = min((tile % n_tiles) * 256 + group * 128 + row, p.N - 1);
      if (p.x_scale != nullptr) xs_next = __ldg(p.x_scale + m);
      if (p.w_scale != nullptr) ws_next = __ldg(p.w_scale + n);
      if (p.bias != nullptr) bias_next = __ldg(p.bias + n);
    };
    fetch_vectors(pair);
    if (res && issuer) fetch_residual(pair, 0, 0);
    for (int tile = pair; tile < total; tile += n_pairs, ++local) {
      const int m0 = (tile / n_tiles) * 256 + (int)rank * 128, n0 = (tile % n_tiles) * 256 + group * 128;
      const int ab = local & 1;
      const float xs = xs_next;
      // read behind the first chunk's barrier; the previous tile's readers are past its last one
      col_s[group * 128 + row] = ws_next;
      col_s[256 + group * 128 + row] = bias_next;
      fetch_vectors(tile + n_pairs);
      // a group goes on or stops as one, whatever a warp's own wait saw: the barriers below count on all four
      if (!tc::named_bar_and(1 + group, 128, tc::mbar_wait_cluster(acc_full + ab, (local >> 1) & 1, abort_flag))) break;
      tc::tc_fence_after();
      const uint32_t t_acc = tmem_base + (uint32_t)(ab * 256 + group * 128) + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
      for (int c = 0; c < kChunks; ++c, ++g) {
        uint8_t* buf = bufs + (g & 1) * kAPStaging;
        uint32_t r[kCols / 32][32];
#pragma unroll
        for (int h = 0; h < kCols / 32; ++h) tc::tmem_ld32(t_acc + (uint32_t)(c * kCols + h * 32), r[h]);
        if (issuer) {
          if (res) {
            tc::bulk_wait_read<0>();                       // the last store has been read out of the other buffer
            if (c + 1 < kChunks) fetch_residual(tile, c + 1, g + 1); else fetch_residual(tile + n_pairs, 0, g + 1);
          } else {
            tc::bulk_wait_read<1>();                       // the store that last used `buf` has been read out of it
          }
        }
        tc::named_bar_sync(1 + group, 128);
        if (res) tc::mbar_wait(res_full + 2 * group + (g & 1), (g >> 1) & 1, abort_flag);   // (gives up: the tile is lost, as reported)
        tc::tmem_ld_wait();
        if (c == kChunks - 1) {                            // accumulator fully read: hand it back to the issuer
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (rank == 0) tc::mbar_arrive(acc_empty + ab);
            else tc::mbar_arrive_remote(acc_empty + ab, 0);
          }
        }
        uint4* my_row = reinterpret_cast<uint4*>(buf + row * 128);
        const float* ws = col_s + group * 128 + c * kCols;
        const float* bb = ws + 256;
        constexpr int kPiece = F32 ? 4 : 8;                // elements of 16 bytes
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v[kPiece];
#pragma unroll
          for (int e = 0; e < kPiece; e += 4) {
            const int i = kPiece * j + e;
            const float4 s4 = *reinterpret_cast<const float4*>(ws + i), b4 = *reinterpret_cast<const float4*>(bb + i);
            const uint32_t* a = &r[i >> 5][i & 31];
            v[e] = act_of(fmaf(__uint_as_float(a[0]) * xs, s4.x, b4.x), p.act);
            v[e + 1] = act_of(fmaf(__uint_as_float(a[1]) * xs, s4.y, b4.y), p.act);
            v[e + 2] = act_of(fmaf(__uint_as_float(a[2]) * xs, s4.z, b4.z), p.act);
            v[e + 3] = act_of(fmaf(__uint_as_float(a[3]) * xs, s4.w, b4.w), p.act);
          }
          uint4* at = my_row + (j ^ (row & 7));
          if (res) {
            const uint4 t = *at;
            const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (F32) v[e] += __uint_as_float(w[e]);
              else { v[(2 * e) % kPiece] += bf16_lo(w[e]); v[(2 * e + 1) % kPiece] += bf16_hi(w[e]); }
            }
          }
          if (F32) *at = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
          else *at = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4 % kPiece], v[5 % kPiece]), pack_bf16x2(v[6 % kPiece], v[7 % kPiece]));
        }
        tc::fence_proxy_async_smem();
        tc::named_bar_sync(1 + group, 128);
        if (issuer) {
          if (m0 < p.M && n0 + c * kCols < p.N) tc::tma_store_2d(&map_y, buf, n0 + c * kCols, m0);
          tc::bulk_commit();
        }
      }
    }
    if (issuer) tc::bulk_wait_all();
  }
  // neither CTA may leave while its peer can still read its shared memory or arrive on its barriers
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync_all();
  if (warp == 0) tc::tmem_dealloc_pair(tmem_base, 512);
}

template <bool F8, bool F32, int BN, int STAGES, int SPLIT>
static grace_status_t launch_act(const CUtensorMap& mx, const CUtensorMap& mw, const ActParams& p, cudaStream_t s) {
  using S = ActCfg<BN, STAGES, SPLIT>;
  static unsigned long long attr_set_devices = 0;
  DeviceSetup su(&attr_set_devices);
  if (su) {
    GRACE_CUDA_TRY(cudaFuncSetAttribute(act_kernel<F8, F32, BN, STAGES, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kTotal));
    su.done();
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = SPLIT; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((p.N + BN - 1) / BN * SPLIT, (p.M + kGemmBM - 1) / kGemmBM);
  cfg.blockDim = dim3(kActThreads); cfg.dynamicSmemBytes = S::kTotal; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = SPLIT > 1 ? 2 : 1;
  GRACE_CUDA_TRY(cudaLaunchKernelEx(&cfg, act_kernel<F8, F32, BN, STAGES, SPLIT>, mx, mw, p));
  GRACE_LAUNCH_CHECK();
  return GRACE_OK;
}

template <bool F8, bool F32>
static grace_status_t launch_act_pair(const CUtensorMap& mx, const CUtensorMap& mw, const CUtensorMap& my, const CUtensorMap& mr,
                                      const ActParams& p, cudaStream_t s) {
  static unsigned long long attr_set_devices = 0;
  static int max_clusters_of[kMaxDevices] = {0};
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.blockDim = dim3(kAPThreads); cfg.dynamicSmemBytes = kAPSmem; cfg.stream = s; cfg.attrs = attr; cfg.numAttrs = 2;
  DeviceSetup su(&attr_set_devices);
  if (su) {
    GRACE_CUDA_TRY(cudaFuncSetAttribute(act_pair_kernel<F8, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAPSmem));
    int n_sm = 0, clusters = 0;
    GRACE_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, su.dev));
    cfg.gridDim = dim3(n_sm & ~1);
    GRACE_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, act_pair_kernel<F8, F32>, &cfg));
    if (clusters <= 0) return GRACE_CUDA_ERROR;
    max_clusters_of[su.dev] = clusters < n_sm / 2 ? clusters : n_sm / 2;
    su.done();
  }
  const int64_t total = (int64_t)((p.N + 255) / 256) * ((p.M + 255) / 256);
  const int most = max_clusters_of[su.dev];
  cfg.gridDim = dim3(2 * (unsigned)(total < most ? total : most));
  GRACE_CUDA_TRY(cudaLaunchKernelEx(&cfg, act_pair_kernel<F8, F32>, mx, mw, my, mr, p));
  GRACE_LAUNCH_CHECK();
  return GRACE_OK;
}

template <bool F8, bool F32>
static grace_status_t run_act(const LinearForm& f, const CUtensorMap& mx, const CUtensorMap& mw, const ActParams& p, cudaStream_t s) {
  switch (f.bn * 16 + f.split * 2 + f.per_sm - 1) {
    case 32 * 16 + 2: return launch_act<F8, F32, 32, 8, 1>(mx, mw, p, s);
    case 32 * 16 + 4: return launch_act<F8, F32, 32, 8, 2>(mx, mw, p, s);
    case 64 * 16 + 2: return launch_act<F8, F32, 64, 8, 1>(mx, mw, p, s);
    case 64 * 16 + 4: return launch_act<F8, F32, 64, 8, 2>(mx, mw, p, s);
    case 64 * 16 + 8: return launch_act<F8, F32, 64, 8, 4>(mx, mw, p, s);
    case 128 * 16 + 2: return launch_act<F8, F32, 128, 6, 1>(mx, mw, p, s);
    case 128 * 16 + 4: return launch_act<F8, F32, 128, 4, 2>(mx, mw, p, s);
    case 128 * 16 + 8: return launch_act<F8, F32, 128, 4, 4>(mx, mw, p, s);
    case 64 * 16 + 3: return launch_act<F8, F32, 64, 4, 1>(mx, mw, p, s);
    case 128 * 16 + 3: return launch_act<F8, F32, 128, 3, 1>(mx, mw, p, s);
  }
  return GRACE_UNSUPPORTED_SHAPE;
}

template <bool F8>
static grace_status_t linear_act_impl(const void* x, int64_t ldx, const float* x_scale, const void* w, int64_t ldw, const float* w_scale,
                                      const float* bias, int act, const void* residual, int64_t ldr, uint16_t* y_bf16, float* y_f32,
                                      int64_t ldy, int M, int N, int K, void* stream) {
  constexpr int kEsize = F8 ? 1 : 2, kPer16 = 16 / kEsize, kBK = 128 / kEsize;
  if (!x || !w || ((y_bf16 == nullptr) == (y_f32 == nullptr)) || M <= 0 || N <= 0 || K <= 0) return GRACE_INVALID_ARG;
  if (act < GRACE_ACT_NONE || act > GRACE_ACT_SILU) return GRACE_INVALID_ARG;
  const bool f32 = y_f32 != nullptr;
  const int size = f32 ? 4 : 2;
  void* y = f32 ? (void*)y_f32 : (void*)y_bf16;
  if (!grace_aligned16(x) || !grace_aligned16(w) || (ldx % kPer16) || (ldw % kPer16) || ldx < K || ldw < K || ldy < N ||
      (reinterpret_cast<uintptr_t>(y) % size) || (residual != nullptr && (ldr < N || reinterpret_cast<uintptr_t>(residual) % size)) ||
      (residual == y && ldr != ldy) ||
      ((reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(w_scale) | reinterpret_cast<uintptr_t>(bias)) & 3))
    return GRACE_INVALID_ARG;
  if (K % kPer16) return GRACE_UNSUPPORTED_SHAPE;
  ActParams p;
  p.x_scale = x_scale; p.w_scale = w_scale; p.bias = bias; p.residual = residual; p.y = y;
  p.ldr = ldr; p.ldy = ldy; p.M = M; p.N = N; p.KB = (K + kBK - 1) / kBK; p.act = act;
  cudaStream_t s = (cudaStream_t)stream;
  // The pair kernel moves y and the residual by TMA: rows that start on 16 bytes.
  const bool tma_rows = ((reinterpret_cast<uintptr_t>(y) | (uintptr_t)(ldy * size)) & 15) == 0 &&
                        (residual == nullptr || ((reinterpret_cast<uintptr_t>(residual) | (uintptr_t)(ldr * size)) & 15) == 0);
  const bool pair_possible = linear_pair_possible(M, N, !tma_rows);
  if (!pair_possible && (M + kGemmBM - 1) / kGemmBM > 65535) return GRACE_UNSUPPORTED_SHAPE;
  const LinearForm form = linear_form(M, N, p.KB * kGemmBK, pair_possible, kStatsNone, false);
  const CUtensorMapDataType type = F8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  CUtensorMap mx, mw;
  const uint64_t dx[2] = {(uint64_t)K, (uint64_t)M}, sx[1] = {(uint64_t)ldx}, dw[2] = {(uint64_t)K, (uint64_t)N}, sw[1] = {(uint64_t)ldw};
  const uint32_t bx[2] = {(uint32_t)kBK, 128u}, bw[2] = {(uint32_t)kBK, form.bn == 0 ? 128u : (uint32_t)form.bn};
  if (!tc::make_tmap_typed(&mx, x, 2, dx, sx, bx, type, kEsize) || !tc::make_tmap_typed(&mw, w, 2, dw, sw, bw, type, kEsize)) return GRACE_CUDA_ERROR;
  if (form.bn != 0) return f32 ? run_act<F8, true>(form, mx, mw, p, s) : run_act<F8, false>(form, mx, mw, p, s);
  CUtensorMap my, mr;
  const uint64_t dy[2] = {(uint64_t)N, (uint64_t)M}, sy[1] = {(uint64_t)ldy}, sr[1] = {(uint64_t)ldr};
  const uint32_t by[2] = {f32 ? 32u : 64u, 128u};
  if (!tc::make_tmap(&my, y, 2, dy, sy, by, f32)) return GRACE_CUDA_ERROR;
  mr = my;
  if (residual != nullptr && !tc::make_tmap(&mr, residual, 2, dy, sr, by, f32)) return GRACE_CUDA_ERROR;
  return f32 ? launch_act_pair<F8, true>(mx, mw, my, mr, p, s) : launch_act_pair<F8, false>(mx, mw, my, mr, p, s);
}
int linear_act_tc_timeouts() { return tc::tc_timeouts_read_and_clear(); }

}  // namespace grace

extern "C" grace_status_t grace_linear_act(const uint16_t* x, int64_t ldx, const uint16_t* w, int64_t ldw, const float* bias, int act,
                                           const void* residual, int64_t ldr, uint16_t* y_bf16, float* y_f32, int64_t ldy,
                                           int M, int N, int K, void* stream) {
  return grace::linear_act_impl<false>(x, ldx, nullptr, w, ldw, nullptr, bias, act, residual, ldr, y_bf16, y_f32, ldy, M, N, K, stream);
}

extern "C" grace_status_t grace_linear_act_e4m3(const uint8_t* x, int64_t ldx, const float* x_scale, const uint8_t* w, int64_t ldw,
                                                const float* w_scale, const float* bias, int act, const void* residual, int64_t ldr,
                                                uint16_t* y_bf16, float* y_f32, int64_t ldy, int M, int N, int K, void* stream) {
  return grace::linear_act_impl<true>(x, ldx, x_scale, w, ldw, w_scale, bias, act, residual, ldr, y_bf16, y_f32, ldy, M, N, K, stream);
}
