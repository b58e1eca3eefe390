// y = act(x_scale[m] w_scale[n] (x @ w^T) + bias) + residual on tcgen05 tensor cores, bf16 or e4m3 operands, bf16 or fp32
// output: grace_linear's products with the epilogue that decoders with biases, smooth activations or 8-bit weights need.
//
// A k-block is 128 bytes of a row of either type (64 bf16, 128 e4m3) and four MMAs (K = 16 / K = 32), so both types share
// tiles, swizzle, descriptors and the dispatch rule of linear_form.cuh; an e4m3 product has half the k-blocks.
// act_kernel: one 128 x BN tile per CTA or per cluster that shares its K range.  act_pair_kernel: persistent CTA pairs on
// 256 x 256 tiles, two accumulators in TMEM, the epilogue of one under the products of the other.
#include <algorithm>
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
  int bn;                                                  // act_pair_kernel: columns of a tile
};

__device__ __forceinline__ float act_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float act_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// An epilogue's activations are bound by the MUFU pipe (an exponential or a reciprocal is 8 clocks of a scheduler's, a
// packed fma of two elements one slot), so a pair of elements takes two exponentials and at most one reciprocal:
//   v / (1 + 2^s), v' / (1 + 2^s'): with a = 1 + 2^s, b = 1 + 2^s', r = 1 / (a b):  v b r and v' a r.
// s is held at 60 (2^120 and its reciprocal are fp32 numbers) and v at -64 with it: beyond, the results are above -2^-54.
// (Scalar operations: a packed one of two elements saves a slot, but takes its constants from register pairs, which cost two
// more to fill where registers are short.)
__device__ __forceinline__ void act_over_pair(float& v0, float& v1, float s0, float s1) {
  const float a = act_ex2(fminf(s0, 60.f)) + 1.f, b = act_ex2(fminf(s1, 60.f)) + 1.f;
  const float r = act_rcp(a * b);
  v0 = max_nan(v0, -64.f) * (b * r);
  v1 = max_nan(v1, -64.f) * (a * r);
}
__device__ __forceinline__ void act_silu(float& v0, float& v1) {
  constexpr float kLog2e = 1.4426950408889634f;
  act_over_pair(v0, v1, -kLog2e * v0, -kLog2e * v1);
}
__device__ __forceinline__ void act_gelu_tanh(float& v0, float& v1) {
  // (1 + tanh z) / 2 = 1 / (1 + e^-2z), 2z = sqrt(8 / pi) (v + 0.044715 v^3), times log2(e)
  act_over_pair(v0, v1, v0 * fmaf(v0 * v0, -0.10294324f, -2.3022082f), v1 * fmaf(v1 * v1, -0.10294324f, -2.3022082f));
}
// v Phi(v) = max(v, 0) - a Phi(-a), a = |v|, and Phi(-a) = 2^P(a): log2 Phi(-a) is smooth and nearly quadratic.  P is a fit of it for
// the smallest greatest error (least squares over Chebyshev nodes, reweighted by the error), coefficients rounded to fp32 from the highest on
// and the others fitted again.  Phi(-a) is then off, by fit and roundings (P falls to -63) and the exponential, by less than
//   bf16 results, degree 8 up to a = 9       2^-16 of itself: 1 / 128 of half a bf16 step
//   fp32 results, degree 12 up to a = 8.6    2^-20.3 up to 2, 2^-18.5 up to 5, 2^-15.7 up to 8.6
// From there on a stays, and what is left is above -2^-54.  (1 + erff has no digits left at -5.7; erfcf has, but took 342 us for 65536 x 2048 x 512
// e4m3 to fp32, which takes 172 so and took 213 with erff.)
__device__ __forceinline__ float act_gelu_one_f32(float v) {
  const float a = fminf(fabsf(v), 8.6f);
  float q = fmaf(a, -7.3320009785771134e-11f, 4.0688297175961452e-09f);
  q = fmaf(a, q, -1.0023314445106735e-07f);
  q = fmaf(a, q, 1.4398045777852531e-06f);
  q = fmaf(a, q, -1.3235676306067035e-05f);
  q = fmaf(a, q, 7.87459357525222e-05f);
  q = fmaf(a, q, -0.00026501136017031968f);
  q = fmaf(a, q, -6.315719656413421e-05f);
  q = fmaf(a, q, 0.0070560760796070099f);
  q = fmaf(a, q, -0.052534673362970352f);
  q = fmaf(a, q, -0.45918348431587219f);
  q = fmaf(a, q, -1.1511095762252808f);
  q = fmaf(a, q, -0.99999994039535522f);
  return fmaf(-a, act_ex2(q), max_nan(v, 0.f));
}
__device__ __forceinline__ void act_gelu_f32(float& v0, float& v1) { v0 = act_gelu_one_f32(v0); v1 = act_gelu_one_f32(v1); }
// (packed: 65536 x 2048 x 512 e4m3 152 -> 127 us; rows of y that do not start on 16 bytes, 20000 x 1001 x 1024, 41 -> 43)
__device__ __forceinline__ void act_gelu_bf16(float& v0, float& v1) {
  const float a0 = fminf(fabsf(v0), 9.f), a1 = fminf(fabsf(v1), 9.f);
  const f32x2_t a = f2_pack(a0, a1);
  auto both = [](float c) { return f2_pack(c, c); };
  f32x2_t q = f2_fma(a, both(7.4632509949879022e-08f), both(-3.6557726161845494e-06f));
  q = f2_fma(a, q, both(7.9437530075665563e-05f));
  q = f2_fma(a, q, both(-1.0200483957305551e-03f));
  q = f2_fma(a, q, both(8.7508680298924446e-03f));
  q = f2_fma(a, q, both(-5.4304659366607666e-02f));
  q = f2_fma(a, q, both(-4.5824155211448669e-01f));
  q = f2_fma(a, q, both(-1.1512949466705322f));
  q = f2_fma(a, q, both(-0.9999966025352478f));
  float q0, q1;
  f2_unpack(q, q0, q1);
  v0 = fmaf(-a0, act_ex2(q0), max_nan(v0, 0.f));
  v1 = fmaf(-a1, act_ex2(q1), max_nan(v1, 0.f));
}
// The activation of a whole array: one branch for all of it (one per element is an indirect branch each: 65536 x 2048 x 512
// took 463 us so, without any activation).
template <bool F32, int N>
__device__ __forceinline__ void act_all(float (&v)[N], int act) {
  auto all = [&](auto f) {
#pragma unroll
    for (int i = 0; i < N; i += 2) f(v[i], v[i + 1]);
  };
  switch (act) {
    case GRACE_ACT_RELU: all([](float& x, float& y) { x = max_nan(x, 0.f); y = max_nan(y, 0.f); }); break;
    case GRACE_ACT_GELU: if constexpr (F32) all(act_gelu_f32); else all(act_gelu_bf16); break;
    case GRACE_ACT_GELU_TANH: all(act_gelu_tanh); break;
    case GRACE_ACT_SILU: all(act_silu); break;
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
// The tensor cores' accumulator drops what it cannot hold at every step, towards zero: 6.2e-8 of the result per k-block of four steps
// (root mean square, normal operands), 5e-6 over K = 8192 in this kernel's longest chains, where an fp32 product on the cores
// is off by 5e-7.  So fp32 results of more k-blocks than this are added up segment by segment outside, rounded to nearest: 6.8e-7 at
// 500 x 1000 x 8192 in 16.2 us (segments of 16: 9.97e-7, 15.6 us; of 8: 4.7e-7, 16.5 us).
constexpr int kActSegment = 12;

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
  uint64_t* accum_bar = empty + STAGES;                    // [2]: a segment's products are done
  uint64_t* drained = accum_bar + 2;                       // the row warps have taken a segment behind the first
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  constexpr int kTmemCols = F32 ? 2 * BN : (BN < 32 ? 32 : BN);   // fp32: the sum, and a segment
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = SPLIT > 1 ? (int)(blockIdx.x % SPLIT) : 0;
  const int m0 = blockIdx.y * kGemmBM, n0 = (int)(blockIdx.x / SPLIT) * BN;
  const int kb0 = p.KB * rank / SPLIT, KB = p.KB * (rank + 1) / SPLIT - kb0;             // this CTA's k-blocks (>= 1)

  if (SPLIT > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // "this CTA has started"
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { tc::mbar_init(full + s, 1); tc::mbar_init(empty + s, 1); }
    tc::mbar_init(accum_bar, 1); tc::mbar_init(accum_bar + 1, 1); tc::mbar_init(drained, 4);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 4) {
    if (lane == 0) { tc::tma_prefetch_desc(&map_x); tc::tma_prefetch_desc(&map_w); }
    __syncwarp();
    tc::tmem_alloc(tmem_slot, kTmemCols);
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
      bool issued = true;
      for (int kb0 = 0, seg = 0; issued && kb0 < KB; kb0 += kActSegment, ++seg) {
        const int kb1 = F32 ? min(kb0 + kActSegment, KB) : KB;
        if (F32 && seg >= 2) {
          if (!tc::mbar_wait(drained, seg & 1, abort_flag)) break;
          tc::tc_fence_after();
        }
        const uint32_t d_tmem = tmem_base + (F32 && seg > 0 ? (uint32_t)BN : 0u);
        for (int kb = kb0; kb < kb1; ++kb) {
          const int s = kb % STAGES;
          issued = tc::mbar_wait(full + s, (kb / STAGES) & 1, abort_flag);
          if (!issued) break;
          tc::tc_fence_after();
          const uint32_t a_addr = tc::smem_addr(tiles + s * S::kStageBytes);
          const uint64_t a_desc = tc::smem_desc_sw128(a_addr, 16, 1024);
          const uint64_t b_desc = tc::smem_desc_sw128(a_addr + S::kABytes, 16, 1024);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            act_mma<F8, false>(d_tmem, a_desc + (uint64_t)(2 * k), b_desc + (uint64_t)(2 * k), idesc, (kb > kb0 || k) ? 1u : 0u);
          tc::mma_commit(empty + s);
        }
        tc::mma_commit(accum_bar + (seg & 1));
        if (!F32) break;
      }
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
    if constexpr (F32) {
      const uint32_t sum = tmem_base + ((uint32_t)(warp * 32) << 16);
      for (int seg = 1; ok && seg * kActSegment < KB; ++seg) {
        ok = tc::mbar_wait(accum_bar + (seg & 1), (seg >> 1) & 1, abort_flag);
        ok = __all_sync(kFullMask, ok);
        tc::tc_fence_after();
        if (!ok) break;
#pragma unroll 1
        for (int c = 0; c < BN; c += 32) {
          uint32_t a[2][16], b[2][16];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            tc::tmem_ld16(sum + c + 16 * h, a[h]);
            tc::tmem_ld16(sum + BN + c + 16 * h, b[h]);
          }
          tc::tmem_ld_wait();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 16; ++j) a[h][j] = __float_as_uint(__uint_as_float(a[h][j]) + __uint_as_float(b[h][j]));
            tc::tmem_st16(sum + c + 16 * h, a[h]);
          }
        }
        tc::tmem_st_wait();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(drained);
      }
    }
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
          __syncwarp();                                    // (rows behind the last one store nothing: together again for the load)
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
      __syncwarp();                                        // (rows behind the last one left the turn in front early)
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
        v[j] = fmaf(v[j] * xs, ws.x, bb.x); v[j + 1] = fmaf(v[j + 1] * xs, ws.y, bb.y);
        v[j + 2] = fmaf(v[j + 2] * xs, ws.z, bb.z); v[j + 3] = fmaf(v[j + 3] * xs, ws.w, bb.w);
      }
      act_all<F32>(v, p.act);
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
  if (warp == 4) tc::tmem_dealloc(tmem_base, kTmemCols);
}

// ---------------------------------------------------------------------------------------------
// Persistent CTA pairs: tiles of 256 x bn (n fastest), each CTA with 128 rows of x and bn / 2 of the tile's rows of w in a ring of
// five stages, one tcgen05.mma stream per pair into one of two accumulators (all of TMEM).
// Epilogue: sixteen warps per CTA, each with 32 rows x 64 columns of its own.  A thread has a row: it takes a step's columns
// (32 of a bf16 result, 16 of an fp32 one) out of the accumulator, finishes them and leaves them in the warp's 2 KB of shared
// memory (64 bytes a row, swizzled), from where a TMA store takes them.  The residual comes the same way: row segments into
// registers one step ahead, from there into the 2 KB, and a thread adds its row's where the results will lie.  No warp waits
// for another.  WIDE: rows of y and of the residual start on 16 bytes; otherwise the warp moves single elements between the
// 2 KB and memory.
// LONG (fp32 results of more than kAPSegment k-blocks): an accumulator takes a segment, and the epilogue's warps add them up in
// registers while the other accumulator fills.  Segments of 16 k-blocks leave 1.0e-6 of the result; of 12, 7e-7 for 6 to 22 % more
// time (7003 x 2036 x 8184 with SiLU and residual 278 -> 295 us, 20000 x 1024 x 1024 47 -> 57: the accumulators change hands
// before they are drained); without any, 232 us and 9.1e-6.
// Measured, e4m3 to bf16, L2 flushed between calls: 65536 x 2048 x 512 84 us, with GELU 129, bound by the epilogue's instructions;
// 65536 x 512 x 2048 61.5 us, 2.23 PFLOP/s, 68 with a residual.  (In a row of calls the power limit leaves a lower clock: 140 with GELU, 85
// with a residual, and 324 for 7003 x 2036 x 8184.)
// ---------------------------------------------------------------------------------------------
constexpr int kAPStages = 5;
constexpr int kAPStageBytes = 2 * 128 * 128;
constexpr int kAPWarps = 16, kAPWarpCols = 64;             // columns of a tile that a warp finishes
constexpr int kAPRow = 64;                                 // bytes of a row in a warp's shared memory
constexpr int kAPTurn = 32 * kAPRow;
constexpr int kAPCols = 2 * kAPWarpCols * 4;               // scales and biases of the warp's columns
constexpr int kAPSmem = kAPStages * kAPStageBytes + kAPWarps * (kAPTurn + kAPCols) + 256;
constexpr int kAPThreads = 64 + 32 * kAPWarps;
constexpr int kAPSegment = 16;                              // LONG: k-blocks of an accumulator
static_assert(kAPSmem >= tc::kTmemAllSmem && kAPSmem <= 227 * 1024, "");

// v = acc * xs * scale + bias of N columns, whose scales and biases (kAPWarpCols behind the scales) lie in shared memory.
template <bool F8, int N>
__device__ __forceinline__ void act_affine(float (&v)[N], const uint32_t (&acc)[N], float xs, const float* scale) {
  const f32x2_t x2 = f2_pack(xs, xs);
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 b4 = *reinterpret_cast<const float4*>(scale + kAPWarpCols + i);
    f32x2_t lo = f2_pack(__uint_as_float(acc[i]), __uint_as_float(acc[i + 1])), hi = f2_pack(__uint_as_float(acc[i + 2]), __uint_as_float(acc[i + 3]));
    if (F8) {
      const float4 s4 = *reinterpret_cast<const float4*>(scale + i);
      lo = f2_fma(f2_mul(lo, x2), f2_pack(s4.x, s4.y), f2_pack(b4.x, b4.y));
      hi = f2_fma(f2_mul(hi, x2), f2_pack(s4.z, s4.w), f2_pack(b4.z, b4.w));
    } else {
      lo = f2_add(lo, f2_pack(b4.x, b4.y));
      hi = f2_add(hi, f2_pack(b4.z, b4.w));
    }
    f2_unpack(lo, v[i], v[i + 1]);
    f2_unpack(hi, v[i + 2], v[i + 3]);
  }
}

template <bool F8, bool F32, bool WIDE, bool LONG>
__global__ void __launch_bounds__(kAPThreads, 1)
act_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_y, const ActParams p) {
  extern __shared__ __align__(1024) uint8_t smem_pair[];
  uint8_t* tiles = smem_pair;
  if ((tc::smem_addr(tiles) & 1023u) != 0) {               // the swizzled tiles need it; same answer in every thread
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicAdd(&tc::g_tc_timeouts, 1);
    return;
  }
  uint8_t* turns = tiles + kAPStages * kAPStageBytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(turns + kAPWarps * (kAPTurn + kAPCols));  // even CTA only: both CTAs' bytes landed
  uint64_t* empty = full + kAPStages;                      // the pair's MMAs have read the stage
  uint64_t* acc_full = empty + kAPStages;                  // [2]
  uint64_t* acc_empty = acc_full + 2;                      // [2] even CTA only: the epilogue warps of both
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_cta_rank();            // 0: issues the MMAs; 1: peer
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int n_tiles = (p.N + p.bn - 1) / p.bn, total = n_tiles * ((p.M + 255) / 256);
  constexpr int kBK = F8 ? 128 : 64;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kAPStages; ++s) { tc::mbar_init(full + s, 1); tc::mbar_init(empty + s, 1); }
    for (int a = 0; a < 2; ++a) { tc::mbar_init(acc_full + a, 1); tc::mbar_init(acc_empty + a, 2 * kAPWarps); }
    *abort_flag = 0;
    tc::fence_mbar_init();
    tc::tma_prefetch_desc(&map_x); tc::tma_prefetch_desc(&map_w);
    if (WIDE) tc::tma_prefetch_desc(&map_y);
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
        const int m0 = (tile / n_tiles) * 256 + (int)rank * 128, n0 = (tile % n_tiles) * p.bn + (int)rank * (p.bn / 2);
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const int s = it % kAPStages;
          if (!tc::mbar_wait_cluster(empty + s, ((it / kAPStages) & 1) ^ 1, abort_flag)) { tile = total; break; }
          if (rank == 0) tc::mbar_expect_tx(full + s, 2 * (128 * 128 + p.bn / 2 * 128));   // this CTA's bytes and the peer's
          uint8_t* a = tiles + s * kAPStageBytes;
          const uint32_t bar = tc::cluster_addr_of(full + s, 0);
          tc::tma_load_2d_pair(a, &map_x, bar, kb * kBK, m0);
          tc::tma_load_2d_pair(a + 128 * 128, &map_w, bar, kb * kBK, n0);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {                           // ---- even CTA: MMA issuer for the pair ----
      const uint32_t idesc = act_idesc<F8>(256, p.bn);
      int it = 0, local = 0;
      for (int tile = pair; tile < total; tile += n_pairs) {
        bool ok = true;
        for (int kb0 = 0, kb1; ok && kb0 < p.KB; kb0 = kb1, ++local) {
          const int ab = local & 1;
          kb1 = LONG ? min(kb0 + kAPSegment, p.KB) : p.KB;
          ok = tc::mbar_wait_cluster(acc_empty + ab, ((local >> 1) & 1) ^ 1, abort_flag);
          if (!ok) break;
          tc::tc_fence_after();
          const uint32_t d_tmem = tmem_base + (uint32_t)(ab * 256);
          for (int kb = kb0; kb < kb1; ++kb, ++it) {
            const int s = it % kAPStages;
            ok = tc::mbar_wait_cluster(full + s, (it / kAPStages) & 1, abort_flag);
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t a_addr = tc::smem_addr(tiles + s * kAPStageBytes);
            const uint64_t a_desc = tc::smem_desc_sw128(a_addr, 16, 1024);
            const uint64_t b_desc = tc::smem_desc_sw128(a_addr + 128 * 128, 16, 1024);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              act_mma<F8, true>(d_tmem, a_desc + (uint64_t)(2 * k), b_desc + (uint64_t)(2 * k), idesc, (kb > kb0 || k) ? 1u : 0u);
            tc::mma_commit_pair(empty + s, 3);
          }
          if (ok) tc::mma_commit_pair(acc_full + ab, 3);
        }
        if (!ok) break;
      }
    }
  } else {
    // ---- epilogue warps 2..17: rows q*32 .. of this CTA's 128 (q: the warp's TMEM lane quarter), 64 columns ----
    const int q = warp & 3, col = ((warp - 2) >> 2) * kAPWarpCols;
    constexpr int kSize = F32 ? 4 : 2, kPer = 16 / kSize, kCols = kAPRow / kSize;   // columns of a piece, of a step
    constexpr int kPieces = kAPRow / 16, kRows = 32 / kPieces;  // of a row; rows of 32 pieces
    uint8_t* const turn = turns + (warp - 2) * kAPTurn;     // [32 rows][kPieces], swizzled by the row
    auto piece = [&](int row, int j) { return reinterpret_cast<uint4*>(turn + row * kAPRow + ((j ^ ((row >> 1) & 3)) << 4)); };
    auto element = [&](int row, int c) { return reinterpret_cast<uint8_t*>(piece(row, c / kPer)) + (c % kPer) * kSize; };
    uint4 held[kPieces];                                    // the residual of the next step's columns
    auto hold = [&](int m0, int n0) {
      const int m = m0 + lane / kPieces, n = n0 + lane % kPieces * kPer;
      const char* at = reinterpret_cast<const char*>(p.residual) + ((int64_t)m * p.ldr + n) * kSize;
#pragma unroll
      for (int i = 0; i < kPieces; ++i, at += kRows * p.ldr * kSize) {
        held[i] = make_uint4(0, 0, 0, 0);
        if (m + kRows * i < p.M && n < p.N) {                   // (not .nc: the residual may be y itself)
          if (n + kPer <= p.N) {
            held[i] = *reinterpret_cast<const uint4*>(at);
          } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
              if (n + e >= p.N) continue;
              if (F32) w[e & 3] = reinterpret_cast<const uint32_t*>(at)[e];
              else w[(e >> 1) & 3] |= (uint32_t)reinterpret_cast<const uint16_t*>(at)[e] << (16 * (e & 1));
            }
            held[i] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    };
    // the row's scale and the columns' vectors, one tile ahead; the latter in a copy of the warp's own
    float* const scale = reinterpret_cast<float*>(turns + kAPWarps * kAPTurn + (warp - 2) * kAPCols);
    constexpr int kVec = kAPWarpCols / 32;
    float xs_next, ws_next[kVec], bias_next[kVec];
    auto fetch = [&](int m0, int n0) {
      xs_next = F8 && p.x_scale != nullptr ? __ldg(p.x_scale + min(m0 + lane, p.M - 1)) : 1.f;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const int n = min(n0 + 32 * i + lane, p.N - 1);
        ws_next[i] = F8 && p.w_scale != nullptr ? __ldg(p.w_scale + n) : 1.f;
        bias_next[i] = p.bias != nullptr ? __ldg(p.bias + n) : 0.f;
      }
    };
    int local = 0;                                          // accumulators so far
    // the accumulator: waits for it (false: it will not come), and gives it back
    auto wait_full = [&]() {
      bool ok = tc::mbar_wait_cluster(acc_full + (local & 1), (local >> 1) & 1, abort_flag);
      ok = __all_sync(kFullMask, ok);
      tc::tc_fence_after();
      return ok;
    };
    auto give_back = [&]() {
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (rank == 0) tc::mbar_arrive(acc_empty + (local & 1));
        else tc::mbar_arrive_remote(acc_empty + (local & 1), 0);
      }
      ++local;
    };
    auto t_acc = [&]() { return tmem_base + (uint32_t)((local & 1) * 256 + col) + ((uint32_t)(q * 32) << 16); };
    // the next tile's coordinates without a division
    const int step_m = n_pairs / n_tiles, step_n = n_pairs % n_tiles;
    int tile_m = pair / n_tiles, tile_n = pair % n_tiles;
    int m0 = tile_m * 256 + (int)rank * 128 + q * 32, n0 = tile_n * p.bn + col;
    if (!LONG) fetch(m0, n0);
    for (int tile = pair; tile < total; tile += n_pairs) {
      if constexpr (LONG) {
        // All segments but the last into registers; with the last they go back into its accumulator, and on as one.  (64 of a
        // thread's 96 registers: nothing of the finish is fetched ahead, and the accumulator is read by eights.  What does not fit
        // goes to the L2 and back, the shared memory having left no L1.)
        float sum[kAPWarpCols / 8][8];
        bool ok = true;
        for (int kb0 = 0; kb0 < p.KB; kb0 += kAPSegment) {
          ok = wait_full();
          if (!ok) break;
          const uint32_t t = t_acc();
          const bool last = kb0 + kAPSegment >= p.KB;
#pragma unroll
          for (int c = 0; c < kAPWarpCols / 8; ++c) {
            uint32_t r[8];
            tc::tmem_ld8(t + c * 8, r);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              sum[c][i] = kb0 == 0 ? __uint_as_float(r[i]) : sum[c][i] + __uint_as_float(r[i]);
              r[i] = __float_as_uint(sum[c][i]);
            }
            if (last) tc::tmem_st8(t + c * 8, r);
          }
          if (!last) give_back();
        }
        if (!ok) break;
        tc::tmem_st_wait();
        m0 = tile / n_tiles * 256 + (int)rank * 128 + q * 32;
        n0 = tile % n_tiles * p.bn + col;
        fetch(m0, n0);
      } else {
        m0 = tile_m * 256 + (int)rank * 128 + q * 32;
        n0 = tile_n * p.bn + col;
        tile_m += step_m;
        tile_n += step_n;
        if (tile_n >= n_tiles) { tile_n -= n_tiles; ++tile_m; }
      }
      if (WIDE && p.residual != nullptr) hold(m0, n0);
      const float xs = xs_next;
      __syncwarp();                                         // the tile in front has been finished with them
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (F8) scale[32 * i + lane] = ws_next[i];
        scale[kAPWarpCols + 32 * i + lane] = bias_next[i];
      }
      __syncwarp();                                         // every lane reads all of them
      if (!LONG) fetch(tile_m * 256 + (int)rank * 128 + q * 32, tile_n * p.bn + col);
      // the finished columns c0 .. of the tile: scales, bias, activation, residual, and out
      auto finish = [&](const int c0, const uint32_t (&r)[kCols]) {
        if (m0 >= p.M || n0 + c0 >= p.N || col + c0 >= p.bn) return;               // the same for the whole warp
        float v[kCols];
        act_affine<F8>(v, r, xs, scale + c0);
        act_all<F32>(v, p.act);
        if (WIDE) {
          if (lane == 0) tc::bulk_wait_read<0>();           // the step in front has left the 2 KB
        }
        __syncwarp();
        if (p.residual != nullptr) {
          if (WIDE) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) *piece(kRows * i + lane / kPieces, lane % kPieces) = held[i];
            if (c0 + kCols < kAPWarpCols) hold(m0, n0 + c0 + kCols);
          } else {
            const int c = lane % kCols, rows = min(32, p.M - m0);
            if (n0 + c0 + c < p.N) {
              const char* at = reinterpret_cast<const char*>(p.residual) + ((int64_t)(m0 + lane / kCols) * p.ldr + n0 + c0 + c) * kSize;
#pragma unroll 8
              for (int row = lane / kCols; row < rows; row += 32 / kCols, at += (32 / kCols) * p.ldr * kSize) {
                if (F32) *reinterpret_cast<uint32_t*>(element(row, c)) = *reinterpret_cast<const uint32_t*>(at);
                else *reinterpret_cast<uint16_t*>(element(row, c)) = *reinterpret_cast<const uint16_t*>(at);
              }
            }
          }
          __syncwarp();
        }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          uint4* at = piece(lane, j);
          float* e = v + kPer * j;
          if (p.residual != nullptr) {
            const uint4 t = *at;
            const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if constexpr (F32) e[i] += __uint_as_float(w[i]);
              else { e[2 * i] += bf16_lo(w[i]); e[2 * i + 1] += bf16_hi(w[i]); }
            }
          }
          if constexpr (F32) *at = make_uint4(__float_as_uint(e[0]), __float_as_uint(e[1]), __float_as_uint(e[2]), __float_as_uint(e[3]));
          else *at = make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7]));
        }
        if (WIDE) {
          tc::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tc::tma_store_2d(&map_y, turn, n0 + c0, m0);
            tc::bulk_commit();
          }
        } else {
          __syncwarp();
          const int c = lane % kCols, rows = min(32, p.M - m0);
          if (n0 + c0 + c < p.N) {
            char* at = reinterpret_cast<char*>(p.y) + ((int64_t)(m0 + lane / kCols) * p.ldy + n0 + c0 + c) * kSize;
#pragma unroll 8
            for (int row = lane / kCols; row < rows; row += 32 / kCols, at += (32 / kCols) * p.ldy * kSize) {
              if (F32) *reinterpret_cast<uint32_t*>(at) = *reinterpret_cast<const uint32_t*>(element(row, c));
              else *reinterpret_cast<uint16_t*>(at) = *reinterpret_cast<const uint16_t*>(element(row, c));
            }
          }
        }
      };
      if (!LONG && !wait_full()) break;
      const uint32_t t = t_acc();
#pragma unroll 1
      for (int c0 = 0; c0 < kAPWarpCols; c0 += kCols) {
        uint32_t r[kCols];
        __syncwarp();                                       // (lanes part in the step in front's stores)
        if constexpr (F32) tc::tmem_ld16(t + c0, r); else tc::tmem_ld32(t + c0, r);
        tc::tmem_ld_wait();
        if (c0 + kCols == kAPWarpCols) give_back();         // this part of the accumulator has been read
        finish(c0, r);
      }
    }
    if (WIDE && lane == 0) tc::bulk_wait_all();
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

template <bool F8, bool F32, bool WIDE, bool LONG = false>
static grace_status_t launch_act_pair(const CUtensorMap& mx, const CUtensorMap& mw, const CUtensorMap& my, const ActParams& p, cudaStream_t s) {
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
    GRACE_CUDA_TRY(cudaFuncSetAttribute(act_pair_kernel<F8, F32, WIDE, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAPSmem));
    int n_sm = 0, clusters = 0;
    GRACE_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, su.dev));
    cfg.gridDim = dim3(n_sm & ~1);
    GRACE_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, act_pair_kernel<F8, F32, WIDE, LONG>, &cfg));
    if (clusters <= 0) return GRACE_CUDA_ERROR;
    max_clusters_of[su.dev] = clusters < n_sm / 2 ? clusters : n_sm / 2;
    su.done();
  }
  const int64_t total = (int64_t)((p.N + p.bn - 1) / p.bn) * ((p.M + 255) / 256);
  const int most = max_clusters_of[su.dev];
  cfg.gridDim = dim3(2 * (unsigned)(total < most ? total : most));
  GRACE_CUDA_TRY(cudaLaunchKernelEx(&cfg, act_pair_kernel<F8, F32, WIDE, LONG>, mx, mw, my, p));
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

// Columns of the CTA pairs' tiles: a narrower tile where fewer of the last wave's pairs then stay without one.  A k-block of a
// tile takes 256 + bn clocks (16 KB of x and 64 bn bytes of w through a port of 64 bytes a clock), its epilogue about 6400 whatever bn
// (a warp has 64 columns or none); whichever is more, times the waves.  (Taken in turn, 256 columns and these:
// 6000 x 1100 x 4096 bf16 52.3 -> 49.2 us, 9000 x 777 x 4096 52.9 -> 50.3, 10000 x 512 x 8192 89.0 -> 87.6; a loss of 1.5 % at
// 7003 x 2036 x 8184, 233.7 -> 237.3, where the clock gives way to the power limit.)
static int act_pair_columns(int M, int N, int KB) {
  int best = 256;
  int64_t least = INT64_MAX;
  for (int bn = 256; bn >= 128; bn -= 32) {
    const int64_t tiles = (int64_t)((M + 255) / 256) * ((N + bn - 1) / bn), waves = (tiles + kSmsInTwos / 2 - 1) / (kSmsInTwos / 2);
    const int64_t one = std::max((int64_t)KB * (256 + bn), (int64_t)6400), t = waves * one;
    if (t < least) { least = t; best = bn; }
  }
  return best;
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
  // (tiles' ends are int; without columns for the persistent kernel, row tiles are gridDim.y)
  constexpr int kMost = 0x7fffffff - 255;
  if (K % kPer16 || M > kMost || N > kMost || K > kMost || (!linear_pair_possible(M, N, false) && M > 65535 * kGemmBM)) return GRACE_UNSUPPORTED_SHAPE;
  ActParams p;
  p.x_scale = x_scale; p.w_scale = w_scale; p.bias = bias; p.residual = residual; p.y = y;
  p.ldr = ldr; p.ldy = ldy; p.M = M; p.N = N; p.KB = (K + kBK - 1) / kBK; p.act = act;
  cudaStream_t s = (cudaStream_t)stream;
  const LinearForm form = linear_form(M, N, p.KB * kGemmBK, linear_pair_possible(M, N, false), kStatsNone, false);
  const CUtensorMapDataType type = F8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  CUtensorMap mx, mw;
  const uint64_t dx[2] = {(uint64_t)K, (uint64_t)M}, sx[1] = {(uint64_t)ldx}, dw[2] = {(uint64_t)K, (uint64_t)N}, sw[1] = {(uint64_t)ldw};
  p.bn = act_pair_columns(M, N, p.KB);
  const uint32_t bx[2] = {(uint32_t)kBK, 128u}, bw[2] = {(uint32_t)kBK, form.bn == 0 ? (uint32_t)p.bn / 2 : (uint32_t)form.bn};
  if (!tc::make_tmap_typed(&mx, x, 2, dx, sx, bx, type, kEsize) || !tc::make_tmap_typed(&mw, w, 2, dw, sw, bw, type, kEsize)) return GRACE_CUDA_ERROR;
  if (form.bn != 0) return f32 ? run_act<F8, true>(form, mx, mw, p, s) : run_act<F8, false>(form, mx, mw, p, s);
  const bool wide = ((reinterpret_cast<uintptr_t>(y) | (uintptr_t)(ldy * size)) & 15) == 0 &&
                    (residual == nullptr || ((reinterpret_cast<uintptr_t>(residual) | (uintptr_t)(ldr * size)) & 15) == 0);
  CUtensorMap my = mx;                                     // read with `wide` alone
  const uint64_t dy[2] = {(uint64_t)N, (uint64_t)M}, sy[1] = {(uint64_t)ldy};
  const uint32_t by[2] = {(uint32_t)(kAPRow / size), 32u};
  if (wide && !tc::make_tmap_typed(&my, y, 2, dy, sy, by, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, size,
                                   CU_TENSOR_MAP_SWIZZLE_64B))
    return GRACE_CUDA_ERROR;
  if (f32 && p.KB > kAPSegment)
    return wide ? launch_act_pair<F8, true, true, true>(mx, mw, my, p, s) : launch_act_pair<F8, true, false, true>(mx, mw, my, p, s);
  if (f32) return wide ? launch_act_pair<F8, true, true>(mx, mw, my, p, s) : launch_act_pair<F8, true, false>(mx, mw, my, p, s);
  return wide ? launch_act_pair<F8, false, true>(mx, mw, my, p, s) : launch_act_pair<F8, false, false>(mx, mw, my, p, s);
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
