// Root-mean-square norm of the residual stream with the addition of a block's output on the way, to bf16 or to e4m3 with
// one scale per row (the operand of grace_linear_act_e4m3):
//   s = x + delta (kept, rounded to the stream's type);  n = s * rsqrt(mean(s^2) + eps) * gamma
//   bf16: y = n;   e4m3: scale = max(max|n|, 2^-100) / 448, y = n / scale
// One pass over memory: the row stays in registers as fp32 between the sum of squares, the largest magnitude and the stores,
// so a call reads x, delta and gamma once and writes the stream and y once.  Bound by HBM: 65536 x 512 bf16 with delta to e4m3
// (235 MB) 37.1 us, 6.3 TB/s; 8191 x 2048 fp32 to bf16 (201 MB) 34 us in a row of calls, 5.9 TB/s.
#include <cuda_fp8.h>
#include "common.cuh"

namespace grace {

struct RmsParams {
  const void* x;                 // fp32 or bf16, row stride ldx
  const uint16_t* delta;         // bf16 or NULL
  void* x_out;                   // with delta: the stream's new rows (may be x itself)
  const float* gamma;
  void* y;                       // bf16 or e4m3
  float* scale;                  // e4m3: [R]
  int64_t ldx, ldd, ldxo, ldy;
  int R, D;
  float eps;
};

// A plain 16-byte load that does not stay in L1; not .nc: x_out may be x.
__device__ __forceinline__ uint4 ld_once_u4(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float bf16_round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// NT threads hold a row in pieces of eight elements, PIECES each; VEC: whole 16-byte accesses (every row of every tensor
// 16-byte aligned, D a multiple of 8), otherwise element by element with neighbouring threads on neighbouring elements.
template <bool F32, bool E4M3, bool VEC, int NT, int PIECES>
__global__ void __launch_bounds__(NT < 128 ? 128 : NT)
rms_norm_kernel(const RmsParams p) {
  pdl_wait();
  pdl_trigger();
  constexpr int kRows = NT < 128 ? 128 / NT : 1;           // rows of a CTA
  const int tid = NT < 128 ? threadIdx.x % NT : threadIdx.x;
  const int r = blockIdx.x * kRows + (NT < 128 ? threadIdx.x / NT : 0);
  if (r >= p.R) return;                                    // a warp's rows are whole: NT >= 32
  const int n8 = VEC ? p.D >> 3 : 0;
  auto at = [&](int i, int e) { return VEC ? ((i * NT + tid) << 3) + e : (i * 8 + e) * NT + tid; };

  float v[PIECES][8];
  const char* xrow = reinterpret_cast<const char*>(p.x) + (int64_t)r * p.ldx * (F32 ? 4 : 2);
  const uint16_t* drow = p.delta != nullptr ? p.delta + (int64_t)r * p.ldd : nullptr;
  char* orow = reinterpret_cast<char*>(p.x_out) + (int64_t)r * p.ldxo * (F32 ? 4 : 2);
  if (VEC) {
    uint4 a[PIECES][F32 ? 2 : 1], d[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = i * NT + tid;
      const bool in = c < n8;
#pragma unroll
      for (int h = 0; h < (F32 ? 2 : 1); ++h) a[i][h] = in ? ld_once_u4(xrow + (int64_t)c * (F32 ? 32 : 16) + 16 * h) : make_uint4(0, 0, 0, 0);
      d[i] = in && drow != nullptr ? ld_stream_u4(reinterpret_cast<const uint4*>(drow) + c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const uint32_t dw[4] = {d[i].x, d[i].y, d[i].z, d[i].w};
      if (F32) {
        const uint32_t w[8] = {a[i][0].x, a[i][0].y, a[i][0].z, a[i][0].w, a[i][F32].x, a[i][F32].y, a[i][F32].z, a[i][F32].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = __uint_as_float(w[e]);
      } else {
        const uint32_t w[4] = {a[i][0].x, a[i][0].y, a[i][0].z, a[i][0].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[i][2 * e] = bf16_lo(w[e]); v[i][2 * e + 1] = bf16_hi(w[e]); }
      }
      if (drow != nullptr) {
        const int c = i * NT + tid;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[i][2 * e] += bf16_lo(dw[e]); v[i][2 * e + 1] += bf16_hi(dw[e]); }
        if (F32) {
          if (c < n8) {
            float4* o = reinterpret_cast<float4*>(orow) + 2 * c;
            o[0] = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
            o[1] = make_float4(v[i][4], v[i][5], v[i][6], v[i][7]);
          }
        } else {
          // the norm is that of the stream as it is stored: adding and norming in one call or in two gives the same bits
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16x2(v[i][2 * e], v[i][2 * e + 1]);
            v[i][2 * e] = bf16_lo(w[e]);
            v[i][2 * e + 1] = bf16_hi(w[e]);
          }
          if (c < n8) reinterpret_cast<uint4*>(orow)[c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = at(i, e);
        v[i][e] = 0.f;
        if (j < p.D) {
          float t = F32 ? reinterpret_cast<const float*>(xrow)[j] : __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(xrow)[j] << 16);
          if (drow != nullptr) {
            t += __uint_as_float((uint32_t)drow[j] << 16);
            if (F32) {
              reinterpret_cast<float*>(orow)[j] = t;
            } else {
              t = bf16_round(t);
              reinterpret_cast<uint16_t*>(orow)[j] = (uint16_t)(__float_as_uint(t) >> 16);
            }
          }
          v[i][e] = t;
        }
      }
    }
  }

  __shared__ float red[2][NT / 32];
  auto reduce = [&](float t, int which) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float u = __shfl_xor_sync(kFullMask, t, o);
      t = which == 0 ? t + u : max_nan(t, u);
    }
    if (NT > 32) {
      if ((tid & 31) == 0) red[which][tid >> 5] = t;
      __syncthreads();
      t = red[which][0];
#pragma unroll
      for (int w = 1; w < NT / 32; ++w) t = which == 0 ? t + red[which][w] : max_nan(t, red[which][w]);
    }
    return t;
  };
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) t = fmaf(v[i][e], v[i][e], t);
    sq += t;
  }
  const float rstd = rsqrtf(reduce(sq, 0) / (float)p.D + p.eps);

  float most = 0.f;                                        // NaN with any: a row's scale then says so
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    if (VEC) {
      const int c = i * NT + tid;
      if (c < n8) {
        const float4 g0 = __ldg(reinterpret_cast<const float4*>(p.gamma) + 2 * c), g1 = __ldg(reinterpret_cast<const float4*>(p.gamma) + 2 * c + 1);
        const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * rstd * g[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = at(i, e);
        if (j < p.D) v[i][e] = v[i][e] * rstd * __ldg(p.gamma + j);
      }
    }
    if (E4M3) {
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max_nan(most, fabsf(v[i][e]));
    }
  }

  if (E4M3) {
    // (a row of zeros gets zeros and the least scale, whose reciprocal is an fp32 number)
    most = max_nan(reduce(most, 1), 0x1p-100f);
    const float scale = most / 448.f;
    if (tid == 0) p.scale[r] = scale;
    // n / scale by the reciprocal and the quotient's remainder (Markstein's correction): the fp32 quotient, so that values next to one of
    // e4m3's borders go as the definition has them.  65536 x 512: 39.3 us, by the reciprocal alone 38.9, by divisions 42.3.  (An infinite
    // scale times 0 is left out: its reciprocal is 0, and so is what it divides.)
    const float inv = 1.f / scale, take = isinf(scale) ? 0.f : scale;
    auto over = [&](float n) {
      const float q = n * inv;
      return fmaf(fmaf(-take, q, n), inv, q);
    };
    uint8_t* yrow = reinterpret_cast<uint8_t*>(p.y) + (int64_t)r * p.ldy;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      uint32_t q[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        q[e >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(over(v[i][2 * e]), over(v[i][2 * e + 1])), __NV_SATFINITE, __NV_E4M3) << (16 * (e & 1));
      if (VEC) {
        const int c = i * NT + tid;
        if (c < n8) reinterpret_cast<uint2*>(yrow)[c] = make_uint2(q[0], q[1]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at(i, e) < p.D) yrow[at(i, e)] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
      }
    }
  } else {
    uint16_t* yrow = reinterpret_cast<uint16_t*>(p.y) + (int64_t)r * p.ldy;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(v[i][2 * e], v[i][2 * e + 1]);
      if (VEC) {
        const int c = i * NT + tid;
        if (c < n8) reinterpret_cast<uint4*>(yrow)[c] = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at(i, e) < p.D) yrow[at(i, e)] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

constexpr int kRmsMostD = 16384;
// A warp has up to 1024 elements of a row (32 registers a thread: no barrier, four rows in flight a CTA), 128 threads up to 4096, 512
// the longest.

template <bool F32, bool E4M3, bool VEC>
static void launch_rms(const RmsParams& p, cudaStream_t s) {
  const int pieces = (p.D + 7) / 8;
  const dim3 four((p.R + 3) / 4), one(p.R);
  if (pieces <= 32) launch_pdl(rms_norm_kernel<F32, E4M3, VEC, 32, 1>, four, dim3(128), 0, s, p);
  else if (pieces <= 64) launch_pdl(rms_norm_kernel<F32, E4M3, VEC, 32, 2>, four, dim3(128), 0, s, p);
  else if (pieces <= 128) launch_pdl(rms_norm_kernel<F32, E4M3, VEC, 32, 4>, four, dim3(128), 0, s, p);
  else if (pieces <= 256) launch_pdl(rms_norm_kernel<F32, E4M3, VEC, 128, 2>, one, dim3(128), 0, s, p);
  else if (pieces <= 512) launch_pdl(rms_norm_kernel<F32, E4M3, VEC, 128, 4>, one, dim3(128), 0, s, p);
  else launch_pdl(rms_norm_kernel<F32, E4M3, VEC, 512, 4>, one, dim3(512), 0, s, p);
}

}  // namespace grace

static bool rms_rows_aligned(const void* p, int64_t ld, int size, int to) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) % to) == 0 && (ld * size) % to == 0);
}

extern "C" grace_status_t grace_rms_norm(const float* x_f32, const uint16_t* x_bf16, int64_t ldx, const uint16_t* delta,
                                         int64_t ld_delta, void* x_out, int64_t ldx_out, const float* gamma,
                                         uint16_t* y_bf16, uint8_t* y_e4m3, int64_t ldy, float* y_scale,
                                         int R, int D, float eps, void* stream) {
  using namespace grace;
  if ((x_f32 == nullptr) == (x_bf16 == nullptr) || (y_bf16 == nullptr) == (y_e4m3 == nullptr) || !gamma) return GRACE_INVALID_ARG;
  if (R <= 0 || D <= 0 || ldx < D || ldy < D || !(eps >= 0.f)) return GRACE_INVALID_ARG;
  if ((delta == nullptr) != (x_out == nullptr) || (y_e4m3 == nullptr) != (y_scale == nullptr)) return GRACE_INVALID_ARG;
  if (delta != nullptr && (ld_delta < D || ldx_out < D)) return GRACE_INVALID_ARG;
  const bool f32 = x_f32 != nullptr;
  const void* x = f32 ? (const void*)x_f32 : (const void*)x_bf16;
  const int size = f32 ? 4 : 2;
  // the elements' own alignment; in place only row by row
  if ((reinterpret_cast<uintptr_t>(x) % size) || (reinterpret_cast<uintptr_t>(x_out) % size) || (reinterpret_cast<uintptr_t>(delta) & 1) ||
      (reinterpret_cast<uintptr_t>(gamma) & 3) || (reinterpret_cast<uintptr_t>(y_bf16) & 1) || (reinterpret_cast<uintptr_t>(y_scale) & 3) ||
      (x_out == x && ldx_out != ldx))
    return GRACE_INVALID_ARG;
  if (D > kRmsMostD || R > 0x7fffffff - 3) return GRACE_UNSUPPORTED_SHAPE;              // (four rows a CTA, counted in int)
  RmsParams p;
  p.x = x; p.delta = delta; p.x_out = x_out; p.gamma = gamma;
  p.y = y_bf16 != nullptr ? (void*)y_bf16 : (void*)y_e4m3;
  p.scale = y_scale; p.ldx = ldx; p.ldd = ld_delta; p.ldxo = ldx_out; p.ldy = ldy; p.R = R; p.D = D; p.eps = eps;
  const bool vec = (D & 7) == 0 && grace_aligned16(gamma) && rms_rows_aligned(x, ldx, size, 16) && rms_rows_aligned(x_out, ldx_out, size, 16) &&
                   rms_rows_aligned(delta, ld_delta, 2, 16) && rms_rows_aligned(y_bf16, ldy, 2, 16) && rms_rows_aligned(y_e4m3, ldy, 1, 8);
  cudaStream_t s = (cudaStream_t)stream;
  switch ((f32 ? 4 : 0) + (y_e4m3 != nullptr ? 2 : 0) + (vec ? 1 : 0)) {
    case 0: launch_rms<false, false, false>(p, s); break;
    case 1: launch_rms<false, false, true>(p, s); break;
    case 2: launch_rms<false, true, false>(p, s); break;
    case 3: launch_rms<false, true, true>(p, s); break;
    case 4: launch_rms<true, false, false>(p, s); break;
    case 5: launch_rms<true, false, true>(p, s); break;
    case 6: launch_rms<true, true, false>(p, s); break;
    default: launch_rms<true, true, true>(p, s); break;
  }
  GRACE_LAUNCH_CHECK();
  return GRACE_OK;
}
