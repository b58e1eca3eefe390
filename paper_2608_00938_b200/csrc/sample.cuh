// Tokens drawn from a row's (allowed) logits: temperature, top-k, top-p, min-p, one uniform number per draw.
//
//   w_v = e^((x_v - max) / T) over the allowed tokens, in the order (x descending, token ascending).  Every limit leaves a
//   prefix of that order, so what is kept is a cut (t, i): tokens with x > t, and of those with x = t the ones up to token i.
//   A draw takes the first kept token, in ascending order, at which the running sum of kept weights exceeds u times the whole.
//
// A warp has a row of up to 2048 tokens, a CTA a longer one (or one of few).  A pass or two over the row leave a list of the
// elements that can be kept: those of at least min-p's bound, of the histogram steps down to the one that holds the top_k-th or top-p's cut, or
// heavy enough for top-p (a set whose weights are all at most (1 - p) S / n weighs at most (1 - p) S, so nothing of it is
// needed to reach p S).  With a constraint the list is the allowed tokens.  Everything else happens on the list, in shared
// memory.  The loops are rolled: unrolled over a row in registers, the same steps waited for instructions six cycles of
// fourteen.
// No sort: the cut is found through a histogram of 256 equal steps of (max - x) / T, in counts (top-k) or in fixed-point
// weights (top-p), whose one step that holds the cut is then resolved value by value.
// Measured (65536 x 2048 fp32, one draw; a read at the rate of a copy takes 82 us): no limit 310 us, T = 0 143, min-p 0.02 225, top-k 50
// 334, top-p 0.9 520, top-p 0.95 with min-p 0.05 395, top-k 200 with top-p 0.95 and min-p 0.02 501; a twentieth allowed, top-p 0.9 175.  Bound by instructions and the latency of dependent ones.
// The answer is that of the definition in 64 bits, at the cost of 32: weights and sums are fp32, every comparison of a sum with
// a border has a margin above the sums' worst error, and a row for which one falls inside the margin is done again with
// e^ and sums in fp64.
#pragma once

#include <type_traits>
#include "common.cuh"

namespace grace {

struct SampleParams {
  const void* logits;            // fp32 or bf16 [R][ld]
  const uint64_t* allow;         // [R][words] or NULL
  const float *row_score, *row_lse;                        // [R] or NULL
  const float* temperature;      // [B] or NULL, as the next three
  const int32_t* top_k;
  const float *top_p, *min_p;
  const float* u;                // [R][draws]
  float *out_score, *out_logq;   // [R][draws]
  int32_t *out_parent, *out_token;
  int32_t* d_status;
  int64_t ld, R;
  int M, V, draws, vec;          // vec: quads of a row lie on their own size
  int cap, tokens_cap;           // elements in a team's shared memory, of a list with tokens (multiples of 16)
  int team_bytes;                // shared memory of a team
};

constexpr int kSampleBuckets = 256;
// Steps of the histogram: 256 over 22 powers of two of weight; the last one holds all that is lighter.
constexpr float kSampleSteps = 256.f / 22.f;
constexpr int kSampleMostV = 65536, kSampleMostDraws = 1 << 30;

__device__ __forceinline__ float sample_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// What weights are and are added up in before 64 bits decide.  A warp's rows are many and short: fp32, and one in some dozens
// is done again.  In a CTA's rows, of up to 65536 tokens, a border is next to some sum nearly always, and the one row that is done
// again holds up the call (64 x 65472, top-p 0.95: 70 us, 28 without): fp64, with an e^ that is good to 2.8e-10.
template <int NW>
using Sum = std::conditional_t<NW == 1, float, double>;
// 2^y for y <= 0 to 2.8e-10 of itself: 2^floor times the Taylor polynomial of degree 8 of 2^f, |f| <= 1/2
// ((ln 2 / 2)^9 / 9! = 2e-10, of 2^-1/2 at the least); 2^-1000 and less come out as about 2^-1000.
__device__ __forceinline__ double sample_ex2_fine(double y) {
  y = fmax(y, -1000.);
  const double magic = 6755399441055744.;                  // 3 x 2^51: the sum's last bits are the nearest integer
  const double r = y + magic, f = y - (r - magic);
  double p = 1.3215486790144305e-6;                        // ln(2)^k / k!
  p = fma(p, f, 1.5252733804059841e-5);
  p = fma(p, f, 1.5403530393381606e-4);
  p = fma(p, f, 1.3333558146428443e-3);
  p = fma(p, f, 9.6181291076284772e-3);
  p = fma(p, f, 5.5504108664821580e-2);
  p = fma(p, f, 2.4022650695910072e-1);
  p = fma(p, f, 6.9314718055994531e-1);
  p = fma(p, f, 1.);
  return __hiloint2double(__double2hiint(p) + (__double2loint(r) << 20), __double2loint(p));
}

// The histogram's step of a value.
__device__ __forceinline__ int sample_bucket(float m, float x, float c) { return min(kSampleBuckets - 1, (int)((m - x) * (c * kSampleSteps))); }
// A weight in 64 bits, for the rows that need them (a function of its own: e^ in 64 bits is long).
static __device__ __noinline__ double sample_weight64(float x, float m, float t) { return exp(((double)x - (double)m) / (double)t); }

// The threads that share a row: a warp, or a CTA.
template <int NW>
struct Team {
  static constexpr int NT = NW * 32;
  int tid;
  double* red;                                             // [NW] shared, NW > 1
  __device__ __forceinline__ void sync() const {
    if (NW == 1) __syncwarp(); else __syncthreads();
  }
  template <class T, class Op>
  __device__ __forceinline__ T reduce(T v, Op op) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kFullMask, v, o));
    if (NW > 1) {
      T* r = reinterpret_cast<T*>(red);
      __syncthreads();
      if ((tid & 31) == 0) r[tid >> 5] = v;
      __syncthreads();
      v = r[(tid & 31) & (NW - 1)];
#pragma unroll
      for (int o = NW / 2; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kFullMask, v, o));
    }
    return v;
  }
  template <class T> __device__ __forceinline__ T sum(T v) const { return reduce(v, [](T a, T b) { return a + b; }); }
  __device__ __forceinline__ int sum(int v) const {
    if (NW == 1) return __reduce_add_sync(kFullMask, v);
    return reduce(v, [](int a, int b) { return a + b; });
  }
  // inclusive prefix sum over the threads
  template <class T>
  __device__ __forceinline__ T scan(T v) const {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T t = __shfl_up_sync(kFullMask, v, o);
      if ((tid & 31) >= o) v += t;
    }
    if (NW > 1) {
      T* r = reinterpret_cast<T*>(red);
      __syncthreads();
      if ((tid & 31) == 31) r[tid >> 5] = v;
      __syncthreads();
      T before = T(0);
      for (int w = 0; w < (tid >> 5); ++w) before += r[w];
      v += before;
    }
    return v;
  }
};

template <bool BF16>
__device__ __forceinline__ float logit_at(const char* row, int token) {
  return BF16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(row) + token) << 16) : __ldg(reinterpret_cast<const float*>(row) + token);
}

// A row's elements in the order of their tokens: in shared memory (`tokens` NULL: element i is token i), ...
struct RowShared {
  static constexpr bool kQuads = false;
  const float* vals;
  const uint16_t* tokens;
  int n;
  __device__ __forceinline__ float at(int i) const { return vals[i]; }
  __device__ __forceinline__ int token(int i) const { return tokens != nullptr ? tokens[i] : i; }
};
// ... or where they are, read again by every pass (out of L2): a row of which more stays than a list takes.
template <bool BF16>
struct RowGlobal {
  static constexpr bool kQuads = true;
  const char* row;
  const uint64_t* allow;
  int n, vec;
  bool inf;                      // the row's largest is +inf: these weigh 1, all others nothing
  __device__ __forceinline__ float shown(float x) const { return inf ? (x == INFINITY ? 0.f : -INFINITY) : x; }
  __device__ __forceinline__ float at(int i) const {
    if (allow != nullptr && !((__ldg(allow + (i >> 6)) >> (i & 63)) & 1ull)) return -INFINITY;
    return shown(logit_at<BF16>(row, i));
  }
  __device__ __forceinline__ int token(int i) const { return i; }
  // elements 4q ..: -inf where they are not allowed or beyond the row
  __device__ __forceinline__ float4 quad(int q) const {
    const int i = q << 2;
    if (allow == nullptr && vec && i + 4 <= n && !inf) return whole_quad(q);
    uint32_t bits = allow != nullptr ? (uint32_t)(__ldg(allow + (i >> 6)) >> (i & 63)) & 15u : 15u;
    if (i + 4 > n) bits &= (1u << (n - i)) - 1u;
    float4 t = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (bits == 0u) return t;
    if (vec && i + 4 <= n) {
      t = whole_quad(q);
    } else {
      if (bits & 1u) t.x = logit_at<BF16>(row, i);
      if (bits & 2u) t.y = logit_at<BF16>(row, i + 1);
      if (bits & 4u) t.z = logit_at<BF16>(row, i + 2);
      if (bits & 8u) t.w = logit_at<BF16>(row, i + 3);
    }
    t.x = (bits & 1u) ? shown(t.x) : -INFINITY;
    t.y = (bits & 2u) ? shown(t.y) : -INFINITY;
    t.z = (bits & 4u) ? shown(t.z) : -INFINITY;
    t.w = (bits & 8u) ? shown(t.w) : -INFINITY;
    return t;
  }
  __device__ __forceinline__ float4 whole_quad(int q) const {
    if (!BF16) return __ldg(reinterpret_cast<const float4*>(row) + q);
    const uint2 w = __ldg(reinterpret_cast<const uint2*>(row) + q);
    return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
  }
};
// The elements of a row that its list leaves out, those below `bound`: their weight in 64 bits.
template <bool BF16>
struct LeftOut {
  RowGlobal<BF16> row;
  float bound;
  template <int NW>
  __device__ __forceinline__ double weight64(const Team<NW> tm, float m, float temperature) const {
    double t = 0.;
#pragma unroll 2
    for (int q = tm.tid; q < (row.n + 3) >> 2; q += NW * 32) {
      const float4 v = row.quad(q);
      const float most = fmaxf(fmaxf(v.x < bound ? v.x : -INFINITY, v.y < bound ? v.y : -INFINITY), fmaxf(v.z < bound ? v.z : -INFINITY, v.w < bound ? v.w : -INFINITY));
      if ((most - m) / temperature < -80.f) continue;      // (lighter than 2^-115 each)
      auto left = [&](float x) { return x < bound ? exp(((double)x - (double)m) / (double)temperature) : 0.; };
      t += (left(v.x) + left(v.y)) + (left(v.z) + left(v.w));
    }
    return tm.sum(t);
  }
};

struct Cut {
  float t;                       // x > t, or x = t and place <= last
  int last;
  __device__ __forceinline__ bool keeps(float x, int place) const { return x > t || (x == t && place <= last); }
};

// A team's shared memory, in front of its elements (vals [cap], tokens [tokens_cap]).
template <int NW>
struct SampleShared {
  static constexpr int kList = NW == 1 ? 64 : 256;         // values of a histogram step that are resolved one by one
  union {
    double table[NW * 128];                                // sums of weights over groups of elements, four groups a thread
    uint32_t hist[kSampleBuckets];
  };
  union {
    double prefix[NW * 32];
    float list[kList];
  };
  double red[NW < 2 ? 2 : NW];
  int n_list, bucket, found, found_r;
  float found_t;
  uint32_t above;
  int found_all, place;
  double above_w;
  int len, copies;
};

// First step at which the histogram's running sum reaches goal(its whole sum) (sh.bucket) and the sum in front of it (sh.above);
// -1 if none does.
template <int NW, class Goal>
__device__ __forceinline__ void find_bucket(const Team<NW>& tm, SampleShared<NW>& sh, Goal goal) {
  if (tm.tid < 32) {
    const int lane = tm.tid;
    const uint4 lo = reinterpret_cast<const uint4*>(sh.hist)[2 * lane], hi = reinterpret_cast<const uint4*>(sh.hist)[2 * lane + 1];
    const uint32_t h[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const uint32_t s = ((h[0] + h[1]) + (h[2] + h[3])) + ((h[4] + h[5]) + (h[6] + h[7]));
    uint32_t incl = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t t = __shfl_up_sync(kFullMask, incl, o);
      if (lane >= o) incl += t;
    }
    const uint32_t target = goal(__shfl_sync(kFullMask, incl, 31));
    const uint32_t reached = __ballot_sync(kFullMask, incl >= target);
    if (reached == 0u) {
      if (lane == 0) sh.bucket = -1;
    } else if (lane == __ffs(reached) - 1) {
      uint32_t run = incl - s, front = run;
      int at = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        run += h[j];
        if (run < target) { at = j + 1; front = run; }
      }
      sh.bucket = 8 * lane + at;
      sh.above = front;
    }
  }
  tm.sync();
}
template <int NW>
__device__ __forceinline__ void clear_hist(const Team<NW>& tm, SampleShared<NW>& sh) {
  for (int i = tm.tid; i < kSampleBuckets / 4; i += NW * 32) reinterpret_cast<uint4*>(sh.hist)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// The exact work on a row (a list, as a rule).  Its steps are functions of their own where they are long, and take it by value:
// an object whose address they had would lie in memory, and every loop would read its members from there.
template <int NW, class Row, class Rest>
struct Sampler {
  Row row;
  Team<NW> tm;
  SampleShared<NW>* shared;
  float m;                       // largest value
  float c;                       // log2(e) / T
  float temperature;
  using W = Sum<NW>;
  double c64;                    // log2(e) / T, for fp64 sums
  int group;                     // elements of a table entry
  // top-p counts elements that the list leaves out: their weight with the list's (0: the row is all there is), and where they are
  W whole_row;
  Rest rest;
  static constexpr int NT = NW * 32;
  static constexpr int kList = SampleShared<NW>::kList;

  __device__ __forceinline__ float rough(float x) const { return sample_ex2((x - m) * c); }
  __device__ __forceinline__ W weight(float x) const {
    if constexpr (NW == 1) return rough(x);
    else return sample_ex2_fine(((double)x - (double)m) * c64);
  }
  __device__ __forceinline__ double weight64(float x) const { return sample_weight64(x, m, temperature); }
  // What a comparison of two sums can be off by at the most, the weights' sum being `whole`.  In fp32 (a warp's rows: at most 2048 tokens, group <= 16),
  // in units of 2^-24 of the whole: `steps` (below) and the weights' own errors, which count once for both sums: the exponent's, 3.5 of z = (max - x) / T
  // (the difference, log2(e) / T, the product), whose mean over the weights is at most ln 2048 - ln whole (a distribution's entropy is at most ln n).
  // The steps: 4 of ex2, and one for each addition that an addend passes at most.
  //   cut    top_p of the whole: 15 + 2 + 5 (sample_dense) or 7 + 7 + 5 (narrow), and the product: 23.  The sum in front: 7 + 7 + 5, and the
  //          list's to it: 20.  The difference, the ties' weight and its quotient: 4.  In all 51.
  //   draw   u of the whole: group - 1 + 3 + 5 (tabulate), and the product: group + 8.  The running sum: group + 7, three entries of the table, and an
  //          element: by a scan of five (pick_together) group + 11 in all, or after up to group others (pick) 2 group + 10.  Two for the
  //          comparisons.  In all 25 + 2 group, 24 + 3 group.
  // In fp64: 2.8e-10 of a weight's (sample_ex2_fine), the rest below 2^-44.
  __device__ __forceinline__ W off_by(float steps, W whole) const {
    if constexpr (NW == 1) return (steps + 2.43f * (11.f - __log2f(whole))) * 0x1p-24f * whole;
    else return 1e-9 * whole;
  }
  __device__ __forceinline__ int bucket_of(float x) const { return sample_bucket(m, x, c); }
  template <class F>
  __device__ __forceinline__ void for_each(F f) const {
#pragma unroll 2
    for (int i = tm.tid; i < row.n; i += NT) f(row.at(i), i);
  }
  // The same where sums are formed (SUMS; else for_each): f(x, place) for eight elements of a thread at a time, then done(): a sum by eights and of the eights
  // passes 8 + n / (8 NT) additions instead of n / NT, which is what its error goes by.
  template <bool SUMS, class F, class Done>
  __device__ __forceinline__ void for_each_by_eights(F f, Done done) const {
    if (!SUMS) {
      for_each(f);
      return;
    }
#pragma unroll 1
    for (int i0 = tm.tid; i0 < row.n; i0 += 8 * NT) {
#pragma unroll 2
      for (int i = i0; i < min(i0 + 8 * NT, row.n); i += NT) f(row.at(i), i);
      done();
    }
  }
  __device__ __forceinline__ void note(float t, int r, int same) const {
    shared->found_t = t; shared->found_r = r; shared->found_all = r == same; shared->found = 1;
  }

  // Narrows `cut` to its first k elements (MASS false), or to the fewest whose weights reach p of the sum of its weights.
  // step >= 0: the histogram's step that holds the k-th, and the number of elements in front of it, are known.
  template <bool MASS>
  __device__ __forceinline__ Cut narrow(const Cut cut, const int k, const float p, const int step, const int step_above) const {
    // fixed point: the sum of any row below 2^32
    const float scale = MASS ? __uint_as_float((uint32_t)(126 + __clz(row.n - 1)) << 23) : 1.f;   // 2^(31 - ceil(log2 n))
    auto share = [&](float x) { return MASS ? __float2uint_rn(rough(x) * scale) : 1u; };
    tm.sync();
    if (tm.tid == 0) { shared->n_list = 0; shared->found = 0; }
    int b = step, n_above = step_above;
    if (MASS || step < 0) {
      clear_hist(tm, *shared);
      tm.sync();
      for_each([&](float x, int place) {
        if (cut.keeps(x, place)) atomicAdd(&shared->hist[bucket_of(x)], share(x));
      });
      tm.sync();
      find_bucket(tm, *shared, [&](uint32_t all) {
        if (!MASS) return (uint32_t)k;
        // within what the histogram holds
        const float want = (whole_row > W(0) ? (float)whole_row * scale : (float)all) * p;
        return min(max(1u, (uint32_t)fminf(want, 4294967040.f)), max(1u, all));
      });
      if (shared->bucket < 0) return cut;                  // no more than k elements
      b = shared->bucket;
      n_above = (int)shared->above;
    } else {
      tm.sync();
    }
    W whole = W(0), above = W(0);
    // the step's values; fixed point may have missed the step by a little: then its neighbour's
    for (int tries = 0; ; ++tries) {
      whole = above = W(0);
      W inside = W(0), whole_8 = W(0), above_8 = W(0);
      for_each_by_eights<MASS>([&](float x, int place) {
        if (!cut.keeps(x, place)) return;
        const int at = bucket_of(x);
        if (MASS) {
          const W w = weight(x);
          whole_8 += w;
          above_8 += at < b ? w : W(0);
          if (NW > 1) inside += at == b ? w : W(0);
        }
        if (at == b) {
          const int i = atomicAdd(&shared->n_list, 1);
          if (i < kList) shared->list[i] = x;
        }
      }, [&]() {
        whole += whole_8;
        above += above_8;
        whole_8 = above_8 = W(0);
      });
      if (MASS) {
        whole = tm.sum(whole);
        if (whole_row > W(0)) {
          // A list that min-p has cut shorter than top-p would: all of it stays, and no border is near.
          if ((W)p * whole_row - whole > off_by(51.f, whole_row)) return cut;
          whole = whole_row;
        }
        above = tm.sum(above);
      }
      tm.sync();
      if (!MASS || NW == 1 || tries == 8) break;
      inside = tm.sum(inside);
      const int move = above > (W)p * whole ? -1 : (above + inside < (W)p * whole ? 1 : 0);
      if (move == 0 || b + move < 0 || b + move >= kSampleBuckets) break;
      b += move;
      tm.sync();
      if (tm.tid == 0) shared->n_list = 0;
      tm.sync();
    }
    const int n = shared->n_list;
    int len = n, copies = 1;
    if (n > kList) {
      narrow_keys<MASS>(*this, cut, k, p, b, scale, whole, above, n_above);
      above = (W)shared->above_w;
      n_above = (int)shared->above;
      len = shared->len;
      copies = shared->copies;
    }
    // The list resolved: the value at which the count or the sum of weights in front passes the goal.
    for (int i = tm.tid; i < len; i += NT) {
      const float x = shared->list[i];
      int same = 0;
      if (MASS) {
        W front = W(0);
        for (int j0 = 0; j0 < len; j0 += 8) {
          W front_8 = W(0);
          for (int j = j0; j < min(j0 + 8, len); ++j) {
            const float y = shared->list[j];
            if (y > x) front_8 += weight(y);
            same += y == x;
          }
          front += front_8;
        }
        front += above;
        same *= copies;
        const W w = weight(x), gap = (W)p * whole - front, slack = off_by(51.f, whole);
        if (gap > slack && gap + slack < w * (W)same) {
          const W q = gap / w, r = ceil(q);
          if (same == 1 || ((r - q) * w > slack && (q - (r - W(1))) * w > slack)) note(x, min(same, max(1, (int)r)), same);
        }
      } else {
        int front = n_above;
        for (int j = 0; j < len; ++j) { const float y = shared->list[j]; front += y > x; same += y == x; }
        same *= copies;
        if (front < k && k <= front + same) note(x, k - front, same);
      }
    }
    tm.sync();
    if (MASS && shared->found == 0) narrow64(*this, cut, p, len, copies);
    Cut out = {shared->found_t, 0x7fffffff};
    if (shared->found_all != 0) {
      if (out.t == cut.t) out.last = cut.last;
      return out;
    }
    out.last = nth_tie(*this, cut, out.t, shared->found_r);
    return out;
  }

  // Place of the r-th of the elements with value t that `cut` keeps.
  static __device__ __noinline__ int nth_tie(const Sampler s, const Cut cut, const float t, const int r) { return s.nth_tie_(cut, t, r); }
  __device__ __forceinline__ int nth_tie_(const Cut cut, const float t, const int r) const {
    int* ties = reinterpret_cast<int*>(shared->list);
    tm.sync();
    if (tm.tid == 0) shared->n_list = 0;
    tm.sync();
    for_each([&](float x, int place) {
      if (x == t && cut.keeps(x, place)) {
        const int i = atomicAdd(&shared->n_list, 1);
        if (i < kList) ties[i] = place;
      }
    });
    tm.sync();
    const int n = shared->n_list;
    if (n <= kList) {
      for (int i = tm.tid; i < n; i += NT) {
        int front = 0;
        for (int j = 0; j < n; ++j) front += ties[j] < ties[i];
        if (front == r - 1) shared->place = ties[i];
      }
      tm.sync();
      return shared->place;
    }
    int lo = 0, hi = row.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      int up_to = 0;
      for_each([&](float x, int place) { up_to += x == t && place <= mid && cut.keeps(x, place); });
      if (tm.sum(up_to) >= r) hi = mid; else lo = mid + 1;
    }
    return lo;
  }

  // A step with more values than the list takes: histograms of equal steps of the ordered bits, until they fit or are all the
  // same (`copies` of one list entry).
  template <bool MASS>
  static __device__ __noinline__ void narrow_keys(const Sampler s, const Cut cut, const int k, const float p, const int b, const float scale, const W whole,
                                                  const W above, const int n_above) {
    s.template narrow_keys_<MASS>(cut, k, p, b, scale, whole, above, n_above);
  }
  template <bool MASS>
  __device__ __forceinline__ void narrow_keys_(const Cut cut, const int k, const float p, const int b, const float scale, const W whole,
                                               W above, int n_above) const {
    uint32_t key_lo = 0xffffffffu, key_hi = 0u;
    for_each([&](float x, int place) {
      if (cut.keeps(x, place) && bucket_of(x) == b) { const uint32_t key = ordered_key(x); key_lo = min(key_lo, key); key_hi = max(key_hi, key); }
    });
    key_lo = tm.reduce(key_lo, [](uint32_t a, uint32_t d) { return min(a, d); });
    key_hi = tm.reduce(key_hi, [](uint32_t a, uint32_t d) { return max(a, d); });
    int n = shared->n_list;
    while (n > kList && key_lo < key_hi) {
      const int shift = max(0, 24 - __clz(key_hi - key_lo));
      tm.sync();
      clear_hist(tm, *shared);
      tm.sync();
      for_each([&](float x, int place) {
        const uint32_t key = ordered_key(x);
        if (key >= key_lo && key <= key_hi && cut.keeps(x, place)) atomicAdd(&shared->hist[(key_hi - key) >> shift], MASS ? __float2uint_rn(rough(x) * scale) : 1u);
      });
      tm.sync();
      find_bucket(tm, *shared, [&](uint32_t all) {
        return MASS ? min((uint32_t)fminf(fmaxf((float)((W)p * whole - above) * scale, 1.f), 4294967040.f), max(1u, all)) : (uint32_t)(k - n_above);
      });
      const int at = max(0, shared->bucket);
      key_hi -= (uint32_t)at << shift;
      key_lo = max(key_lo, key_hi - ((1u << shift) - 1u));
      W more = W(0), more_8 = W(0);
      int inside = 0, over = 0;
      for_each_by_eights<MASS>([&](float x, int place) {
        if (!cut.keeps(x, place)) return;
        const uint32_t key = ordered_key(x);
        if (key > key_hi) { over += 1; if (MASS) more_8 += weight(x); }
        else if (key >= key_lo) inside += 1;
      }, [&]() {
        more += more_8;
        more_8 = W(0);
      });
      n = tm.sum(inside);
      n_above = tm.sum(over);
      if (MASS) above = tm.sum(more);
    }
    tm.sync();
    if (tm.tid == 0) shared->n_list = 0;
    tm.sync();
    const bool one = key_lo == key_hi;
    for_each([&](float x, int place) {
      const uint32_t key = ordered_key(x);
      if (key < key_lo || key > key_hi || !cut.keeps(x, place)) return;
      const int i = one ? 0 : atomicAdd(&shared->n_list, 1);
      if (i < kList) shared->list[i] = x;
    });
    if (tm.tid == 0) {
      shared->above_w = (double)above;
      shared->above = (uint32_t)n_above;
      shared->copies = one ? n : 1;
      shared->len = one ? min(n, 1) : n;
    }
    tm.sync();
  }

  // narrow<true>'s decision by sums in 64 bits: first within the list that 32 bits found, then, should the border lie outside it,
  // by bisection over all values.  Sets shared->found_*.
  static __device__ __noinline__ void narrow64(const Sampler s, const Cut cut, const float p, const int len, const int copies) { s.narrow64_(cut, p, len, copies); }
  __device__ __forceinline__ void narrow64_(const Cut cut, const float p, const int len, const int copies) const {
    // the list in descending order: its sums then do not depend on which thread came first
    constexpr int kPer = (kList + NT - 1) / NT;
    float own[kPer];
    int at[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = tm.tid + e * NT;
      own[e] = i < len ? shared->list[i] : 0.f;
      at[e] = 0;
      for (int j = 0; j < len; ++j) at[e] += shared->list[j] > own[e] || (shared->list[j] == own[e] && j < i);
    }
    tm.sync();
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (tm.tid + e * NT < len) shared->list[at[e]] = own[e];
    tm.sync();
    const float top = len > 0 ? shared->list[0] : -INFINITY;
    double whole = 0., above = 0.;
    for_each([&](float x, int place) {
      if (!cut.keeps(x, place)) return;
      const double w = weight64(x);
      whole += w;
      if (x > top) above += w;
    });
    whole = tm.sum(whole);
    if (whole_row > W(0)) whole += rest.weight64(tm, m, temperature);
    above = tm.sum(above);
    const double goal = (double)p * whole;
    auto settle = [&](float x, double front, int same) {
      note(x, min(same, max(1, (int)fmin(ceil((goal - front) / weight64(x)), 2147483647.))), same);
    };
    // (a value's sum ends where the next one's begins, so one value is found at the most)
    for (int i = tm.tid; i < len; i += NT) {
      const float x = shared->list[i];
      const double w = weight64(x);
      double front = above;
      int j = 0, same = 0;
      for (; shared->list[j] > x; ++j) front += weight64(shared->list[j]);
      double end = front;
      for (; j < len && shared->list[j] == x; ++j, ++same) end += w;
      if (copies > 1) {
        same = copies;
        end = front + w * same;
      }
      if ((front < goal || (front == 0. && goal <= 0.)) && end >= goal) settle(x, front, same);
    }
    tm.sync();
    if (shared->found != 0) return;
    // greatest key whose weights and those of all greater ones reach the goal
    uint32_t lo = kKeyNegInf + 1u, hi = ordered_key(m);
    while (lo < hi) {
      const uint32_t mid = lo + ((hi - lo + 1u) >> 1);
      double reach = 0.;
      for_each([&](float x, int place) { if (ordered_key(x) >= mid && cut.keeps(x, place)) reach += weight64(x); });
      if (tm.sum(reach) >= goal) lo = mid; else hi = mid - 1u;
    }
    double front = 0.;
    int same = 0;
    float least = INFINITY;                                // the kept value at `lo`, or the least kept where rounding reaches none
    for_each([&](float x, int place) {
      if (!cut.keeps(x, place)) return;
      const uint32_t key = ordered_key(x);
      if (key > lo) front += weight64(x);
      same += key == lo;
      if (key >= lo) least = fminf(least, x);
    });
    front = tm.sum(front);
    same = tm.sum(same);
    least = tm.reduce(least, [](float a, float d) { return fminf(a, d); });
    if (tm.tid == 0) {
      if (same > 0) settle(least, front, same);
      else note(least, 1, 1);
    }
    tm.sync();
  }

  // EXACT: in 64 bits throughout
  template <bool EXACT>
  using SumOf = std::conditional_t<EXACT, double, W>;
  template <bool EXACT>
  __device__ __forceinline__ SumOf<EXACT> kept_weight(const Cut cut, float x, int i) const {
    if (!cut.keeps(x, i)) return 0;
    if constexpr (EXACT) return weight64(x);
    else return weight(x);
  }
  template <bool EXACT>
  __device__ __forceinline__ SumOf<EXACT> kept_weight(const Cut cut, int i) const { return kept_weight<EXACT>(cut, row.at(i), i); }
  // The table of sums of the kept weights by groups, and the threads' sums (four groups each) up to and with their own; returns
  // the whole.
  template <bool EXACT>
  __device__ __forceinline__ SumOf<EXACT> tabulate(const Cut cut) const {
    using F = SumOf<EXACT>;
    F* const table = reinterpret_cast<F*>(shared->table);
    tm.sync();
    F s = F(0);
#pragma unroll 1
    for (int e = 0; e < 4; ++e) {
      if (group == 1) {                                    // a short list
        const int i = 4 * tm.tid + e;
        const F t = i < row.n ? kept_weight<EXACT>(cut, i) : F(0);
        table[i] = t;
        s += t;
        continue;
      }
      F t = F(0);
      const int i0 = (4 * tm.tid + e) * group;
      if constexpr (Row::kQuads) {                         // in memory: whole quads
        for (int q = i0 >> 2; q < min(i0 + group, (row.n + 3) & ~3) >> 2; ++q) {
          const float4 v = row.quad(q);
          t += (kept_weight<EXACT>(cut, v.x, 4 * q) + kept_weight<EXACT>(cut, v.y, 4 * q + 1)) +
               (kept_weight<EXACT>(cut, v.z, 4 * q + 2) + kept_weight<EXACT>(cut, v.w, 4 * q + 3));
        }
        table[4 * tm.tid + e] = t;
        s += t;
        continue;
      }
      // each thread from another of its elements on, round once: side by side they would all be on one bank
      int k = tm.tid % group;
      for (int i = 0; i < group; ++i) {
        if (i0 + k < row.n) t += kept_weight<EXACT>(cut, i0 + k);
        k = k + 1 == group ? 0 : k + 1;
      }
      table[4 * tm.tid + e] = t;
      s += t;
    }
    s = tm.scan(s);
    reinterpret_cast<F*>(shared->prefix)[tm.tid] = s;
    tm.sync();
    return reinterpret_cast<const F*>(shared->prefix)[NT - 1];
  }

  // Place of the first kept element at which the running sum exceeds u * whole; `sure` unless a border is within `slack`.
  template <bool EXACT>
  __device__ __forceinline__ int pick(const Cut cut, SumOf<EXACT> whole, float u, SumOf<EXACT> slack, bool& sure) const {
    using F = SumOf<EXACT>;
    const F* const table = reinterpret_cast<const F*>(shared->table);
    const F* prefix = reinterpret_cast<const F*>(shared->prefix);
    const F goal = (F)u * whole;
    int lo = 0, hi = NT - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (prefix[mid] > goal) hi = mid; else lo = mid + 1;
    }
    F run = lo > 0 ? prefix[lo - 1] : F(0);
    sure = false;
    int last = -1;
    // group by group from there on: rounding may leave the border just behind the thread's four
    for (int e = 4 * lo; e < 4 * NT; ++e) {
      const F s = table[e];
      if (run + s <= goal && e + 1 < 4 * NT && (e + 1) * group < row.n) { run += s; continue; }
      for (int i = e * group; i < min((e + 1) * group, row.n); ++i) {
        const F w = kept_weight<EXACT>(cut, i);
        if (w > F(0)) {
          last = i;
          if (run + w > goal) { sure = goal - run > slack && run + w - goal > slack; return i; }
        }
        run += w;
      }
    }
    // u next to 1: the last kept element with a weight
    for (int i = row.n - 1; i >= 0 && last < 0; --i)
      if (kept_weight<EXACT>(cut, i) > F(0)) last = i;
    return last;
  }
  // A draw by sums in 64 bits, for the threads that are not sure (`mine`); `build`: the table does not hold them yet.
  static __device__ __noinline__ int place64(const Sampler s, const Cut cut, const float u, const bool mine, const bool build, const int place) {
    const double whole = build ? s.template tabulate<true>(cut) : s.shared->prefix[NT - 1];
    bool ignored;
    return mine ? s.template pick<true>(cut, whole, u, 0., ignored) : place;
  }
  // The same by a whole warp for one draw (all lanes return it): the lanes take a group's elements at once.
  __device__ __forceinline__ int pick_together(const Cut cut, W whole, float u, W slack, bool& sure) const {
    const W* const prefix = reinterpret_cast<const W*>(shared->prefix);
    const W* const table = reinterpret_cast<const W*>(shared->table);
    const int lane = tm.tid & 31;
    const W goal = (W)u * whole;
    int lo = 0;
    if (NW == 1) {
      const uint32_t over = __ballot_sync(kFullMask, prefix[lane] > goal);
      lo = over != 0u ? __ffs(over) - 1 : 31;
    } else {
      int hi = NT - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] > goal) hi = mid; else lo = mid + 1;
      }
    }
    W run = lo > 0 ? prefix[lo - 1] : W(0);
    int e = 4 * lo;
    while (e < 4 * lo + 3 && run + table[e] <= goal) run += table[e++];
    sure = false;
    for (int i0 = e * group; i0 < min((e + 1) * group, row.n); i0 += 32) {
      const int i = i0 + lane;
      const W w = i < min((e + 1) * group, row.n) ? kept_weight<false>(cut, i) : W(0);
      W upto = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const W v = __shfl_up_sync(kFullMask, upto, o);
        if (lane >= o) upto += v;
      }
      upto += run;
      const uint32_t over = __ballot_sync(kFullMask, w > W(0) && upto > goal);
      if (over != 0u) {
        const int at = __ffs(over) - 1;
        const W after = __shfl_sync(kFullMask, upto, at), own = __shfl_sync(kFullMask, w, at);
        sure = goal - (after - own) > slack && after - goal > slack;
        return i0 + at;
      }
      run = __shfl_sync(kFullMask, upto, 31);
    }
    return 0;                                              // not sure: 64 bits decide
  }
};

// What a row's draws need besides its elements: read before them, so that no trip to memory waits for another.
struct RowLimits {
  float temperature, top_p, min_p;
  int top_k;
  float score, lse, u;           // u: this thread's first draw
  int beam;
  int step = -1, step_above = 0; // top-k: the histogram's step that holds the k-th, where it is known
  float least = -INFINITY;       // min-p's bound on x
};
__device__ __forceinline__ RowLimits row_limits(const SampleParams& p, int64_t r, int tid) {
  const uint32_t b = (uint32_t)r / (uint32_t)p.M;          // (rows are below 2^31)
  RowLimits l;
  l.beam = (int)((uint32_t)r - b * (uint32_t)p.M);
  l.temperature = p.temperature != nullptr ? __ldg(p.temperature + b) : 1.f;
  l.top_k = p.top_k != nullptr ? __ldg(p.top_k + b) : 0;
  l.top_p = p.top_p != nullptr ? __ldg(p.top_p + b) : 1.f;
  l.min_p = p.min_p != nullptr ? __ldg(p.min_p + b) : 0.f;
  l.score = p.row_score != nullptr ? __ldg(p.row_score + r) : 0.f;
  l.lse = p.row_lse != nullptr ? __ldg(p.row_lse + r) : 0.f;
  l.u = tid < p.draws ? __ldg(p.u + r * p.draws + tid) : 0.f;
  return l;
}
struct Scale {                   // of the weights
  float t, c;                    // T, held where log2(e) / T and the histogram's steps of it are fp32 numbers; log2(e) / T
  __device__ __forceinline__ explicit Scale(float temperature) : t(fminf(fmaxf(temperature, 1e-36f), 1e30f)), c(1.44269504f / t) {}
};
// w >= min_p as a bound on x, rounded up to the next fp32.
__device__ __forceinline__ float min_p_bound(float m, float min_p, float t) {
  return min_p < 1.f ? fminf(m, __double2float_ru((double)m + (double)t * log((double)min_p))) : m;
}
// x: the token's logit
__device__ __forceinline__ void store_draw(const SampleParams& p, const RowLimits& l, int64_t r, int d, int token, float x, float logq) {
  const int64_t at = r * p.draws + d;
  p.out_token[at] = token;
  if (p.out_parent != nullptr) p.out_parent[at] = l.beam;
  p.out_score[at] = logq == -INFINITY ? -INFINITY : l.score + (x - l.lse);
  if (p.out_logq != nullptr) p.out_logq[at] = logq;
}
template <int NW>
__device__ __forceinline__ void store_all(const SampleParams& p, const RowLimits& l, const Team<NW>& tm, int64_t r, int token, float x, float logq) {
  for (int d = tm.tid; d < p.draws; d += NW * 32) store_draw(p, l, r, d, token, x, logq);
}

// The limits exactly, on a row that holds all elements they can keep, and the draws.  m: the largest value (finite).
template <int NW, bool BF16, class Row>
__device__ __forceinline__ void limit_and_draw(const SampleParams& p, const Row& row, const Team<NW>& tm, SampleShared<NW>& sh, int64_t r, float m,
                                               const RowLimits& l, const Scale& sc, Sum<NW> whole_row, const LeftOut<BF16>& rest, bool infinite) {
  constexpr int NT = NW * 32;
  using S = Sampler<NW, Row, LeftOut<BF16>>;
  const int quarter = (row.n + 4 * NT - 1) / (4 * NT), group = Row::kQuads ? (quarter + 3) & ~3 : quarter;
  // few draws: a warp together for one after the other; many: each thread its own
  const bool together = p.draws <= 8;
  const S s{row, tm, &sh, m, sc.c, sc.t, NW == 1 ? 0. : 1.4426950408889634 / (double)sc.t, group, whole_row, rest};
  Cut cut = {-INFINITY, -1};
  if (l.top_k > 0 && l.top_k < row.n) cut = s.template narrow<false>(cut, l.top_k, 0.f, l.step, l.step_above);
  if (l.top_p < 1.f) cut = s.template narrow<true>(cut, 0, fmaxf(l.top_p, 0.f), -1, 0);
  if (l.least > cut.t) cut = Cut{l.least, 0x7fffffff};
  const Sum<NW> whole = s.template tabulate<false>(cut), slack = s.off_by((float)(together ? 25 + 2 * group : 24 + 3 * group), whole);
  const float log_whole = logf((float)whole);
  auto store = [&](int d, int place) {
    place = max(place, 0);
    const float x = row.at(place);
    store_draw(p, l, r, d, row.token(place), infinite ? INFINITY : x, (x - m) / sc.t - log_whole);
  };
  bool have64 = false;
  for (int d0 = 0; d0 < p.draws; d0 += together ? 1 : NT) {
    const int d = d0 + (together ? 0 : tm.tid);
    const bool in = d < p.draws && (!together || tm.tid < 32);
    float u = together ? __shfl_sync(kFullMask, l.u, d) : (d0 == 0 ? l.u : (in ? __ldg(p.u + r * p.draws + d) : 0.f));
    u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    bool sure = false;
    int place = -1;
    if (!have64 && in) {
      place = together ? s.pick_together(cut, whole, u, slack, sure) : s.template pick<false>(cut, whole, u, slack, sure);
    }
    const int doubt = tm.reduce(in && !sure ? 1 : 0, [](int a, int e) { return a | e; });
    if (doubt) {
      place = S::place64(s, cut, u, in && !sure && (!together || tm.tid == 0), !have64, place);
      have64 = true;
    }
    if (in && (!together || tm.tid == 0)) store(d, place);
  }
}

// A row without a list yet: dense, or with more allowed tokens than a list takes.  SHARED (one warp): the row lies in the list's
// place and is narrowed there; otherwise every pass reads it.  WHOLE: there is room for all of it when no list holds what stays.
template <int NW, bool BF16, bool SHARED, bool WHOLE>
__device__ __forceinline__ void sample_dense(const SampleParams& p, RowGlobal<BF16> row, const Team<NW>& tm, SampleShared<NW>& sh, float* vals,
                                             uint16_t* tokens, int64_t r, int n, RowLimits l) {
  constexpr int NT = NW * 32;
  const int lane = tm.tid & 31, warp = tm.tid >> 5;
  // a warp's quads are neighbours, lane by lane: `iters` of 32
  const int quads = (p.V + 3) >> 2, iters = (quads + NT - 1) / NT, first = warp * 32 * iters + lane;
  float4* const shared = reinterpret_cast<float4*>(vals);
  auto none = []() { return make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY); };
  // (SHARED: filled up to whole passes with -inf)
  auto quad = [&](int q) { return SHARED ? shared[q] : (q < quads ? row.quad(q) : none()); };
  float m = -INFINITY;
  auto see = [&](const float4& t) { m = max_nan(m, max_nan(max_nan(t.x, t.y), max_nan(t.z, t.w))); };
  int i0 = 0;
  if (row.allow == nullptr && p.vec) {                     // eight loads in flight, of whole quads
    const int whole = min(iters, (p.V / 4 - first + 31) / 32);
    for (; i0 + 8 <= whole; i0 += 8) {
      float4 t[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = row.whole_quad(first + 32 * (i0 + i));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        see(t[i]);
        if (SHARED) shared[first + 32 * (i0 + i)] = t[i];
      }
    }
  }
#pragma unroll 1
  for (; i0 < iters; i0 += 4) {
    float4 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = i0 + i < iters && first + 32 * (i0 + i) < quads ? row.quad(first + 32 * (i0 + i)) : none();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      see(t[i]);
      if (SHARED && i0 + i < iters) shared[first + 32 * (i0 + i)] = t[i];
    }
  }
  m = tm.reduce(m, [](float a, float b) { return max_nan(a, b); });
  if (!(m > -INFINITY)) {                                  // nothing, or NaN
    if (m != m && tm.tid == 0) flag_status(p.d_status, GRACE_DEV_NAN);
    store_all<NW>(p, l, tm, r, 0, 0.f, -INFINITY);
    return;
  }
  // (A thread writes and reads the same quads up to the list, so nothing waits here.)
  if (m == INFINITY) {
    row.inf = true;
    m = 0.f;
    if (SHARED) {
      for (int i = 0; i < iters; ++i) {
        const int q = first + 32 * i;
        const float4 t = shared[q];
        shared[q] = make_float4(row.shown(t.x), row.shown(t.y), row.shown(t.z), row.shown(t.w));
      }
    }
  }
  if (!(l.temperature > 0.f)) {
    int at = 0x7fffffff;
    for (int i = 0; i < iters; ++i) {
      const int q = first + 32 * i;
      const float4 t = quad(q);
      const int j = t.x == m ? 0 : t.y == m ? 1 : t.z == m ? 2 : t.w == m ? 3 : 4;
      if (j < 4) at = min(at, 4 * q + j);
    }
    at = tm.reduce(at, [](int a, int b) { return min(a, b); });
    store_all<NW>(p, l, tm, r, at, row.inf ? INFINITY : m, 0.f);
    return;
  }
  const Scale sc(l.temperature);
  // a bound below which nothing is kept (and nothing counts: top-p's sum is that of the top_k, whatever min-p leaves of them)
  const bool by_count = l.top_k > 0 && l.top_k < n, by_mass = !by_count && l.top_p < 1.f;
  if (l.min_p > 0.f) l.least = min_p_bound(m, l.min_p, sc.t);
  float bound = by_count && l.top_p < 1.f ? -INFINITY : l.least;
  Sum<NW> whole_row = 0;
  // a step's far edge, further by what rounding can make of it
  auto edge = [&](int step) { return m - ((float)(step + 1) * 1.0001f) / (sc.c * kSampleSteps) - fabsf(m) * 0x1p-20f; };
  // top-p: the weights' histogram leaves what is kept and a step or two; the bound on light weights alone, several times that.
  // (65536 x 2048, top-p 0.95 at T = 1.5: 1608 us by the latter, 915 so; 0.9 of bf16 logits 750, 591; 1024 x 16384, top-p
  // 0.9: 159, 144; but top-p 0.9 at T = 1 511, 520, and 0.95 with min-p 0.05, the tighter one, 282, 395.  The longest rows, of which few draw and whose threads meet in the same steps: 64 x 65472, top-p 0.95: 49, 52.)
  constexpr bool kMassHist = NW <= 8;
  if (by_count) {
    clear_hist(tm, sh);
    tm.sync();
    auto count = [&](float x) {
      if (x > -INFINITY) atomicAdd(&sh.hist[sample_bucket(m, x, sc.c)], 1u);
    };
#pragma unroll (SHARED ? 1 : 4)
    for (int i = 0; i < iters; ++i) {
      const float4 t = quad(first + 32 * i);
      count(t.x); count(t.y); count(t.z); count(t.w);
    }
    tm.sync();
    find_bucket(tm, sh, [&](uint32_t) { return (uint32_t)l.top_k; });
    l.step = sh.bucket;
    l.step_above = (int)sh.above;
    if (l.step >= 0 && l.step < kSampleBuckets - 1) bound = fmaxf(bound, edge(l.step));
  } else if (by_mass) {
    Sum<NW> s0 = 0, s1 = 0, s2 = 0, s3 = 0;
    const double c64 = NW == 1 ? 0. : 1.4426950408889634 / (double)sc.t;
    auto weight = [&](float x) -> Sum<NW> {
      if constexpr (NW == 1) return sample_ex2((x - m) * sc.c);
      else return sample_ex2_fine(((double)x - (double)m) * c64);
    };
    // the weights' histogram as well, in fixed point as narrow()'s
    const float scale = __uint_as_float((uint32_t)(126 + __clz(p.V - 1)) << 23);
    if (kMassHist) {
      clear_hist(tm, sh);
      tm.sync();
    }
    auto add = [&](float x, Sum<NW>& sum) {
      const Sum<NW> w = weight(x);
      sum += w;
      if (kMassHist) {
        const uint32_t share = __float2uint_rn((float)w * scale);
        if (share != 0u) atomicAdd(&sh.hist[sample_bucket(m, x, sc.c)], share);
      }
    };
#pragma unroll 2
    for (int i = 0; i < iters; ++i) {
      const float4 t = quad(first + 32 * i);
      add(t.x, s0); add(t.y, s1); add(t.z, s2); add(t.w, s3);
    }
    whole_row = tm.sum((s0 + s1) + (s2 + s3));
    if (kMassHist) {
      // The step at which the running sum has reached top_p of the whole for sure: a share is off by half a unit at most and
      // 2^-18.4 of itself (22 times the roundings of x - m, log2(e) / T and their product).  None where that is beyond the whole:
      // what has less than half a unit is not in it.
      tm.sync();
      find_bucket(tm, sh, [&](uint32_t all) {
        const float want = (float)all * fmaxf(l.top_p, 0.f) * (1.f + 0x1p-16f) + (float)p.V;
        return want < (float)all ? (uint32_t)want : 0xffffffffu;
      });
      if (sh.bucket >= 0 && sh.bucket < kSampleBuckets - 1) bound = fmaxf(bound, edge(sh.bucket));
    }
    const float light = (1.f - fmaxf(l.top_p, 0.f)) * (float)whole_row / (float)n * 0.999f;
    bound = fmaxf(bound, m + log2f(light) / sc.c - 1e-4f / sc.c - fabsf(m) * 0x1p-20f);
  }
  if (by_count || by_mass || l.min_p > 0.f) {
    bound = fmaxf(fminf(bound, m), -3.402823466e38f);      // (-inf is in no list)
    if constexpr (SHARED) {
      // 128 neighbours at a time, in place: the list is never ahead of what has been read.  One that outgrows its tokens' room
      // is given up, and the row read again.
      __syncwarp();
      int kept = 0;
      const uint32_t to_vals = (uint32_t)__cvta_generic_to_shared(vals), to_tokens = (uint32_t)__cvta_generic_to_shared(tokens);
      const uint32_t below = (1u << lane) - 1u;
      auto take = [&](float x, uint32_t& at, int token) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ge.f32 p, %3, %4;\n\t@p st.shared.f32 [%1], %3;\n\t@p st.shared.u16 [%2], %5;\n\t@p add.u32 %0, %0, 1;\n\t}"
                     : "+r"(at) : "r"(to_vals + 4 * at), "r"(to_tokens + 2 * at), "f"(x), "f"(bound), "h"((uint16_t)token) : "memory");
      };
#pragma unroll 2
      for (int i = 0; i < iters; ++i) {
        const float4 t = shared[32 * i + lane];
        const uint32_t b0 = __ballot_sync(kFullMask, t.x >= bound), b1 = __ballot_sync(kFullMask, t.y >= bound), b2 = __ballot_sync(kFullMask, t.z >= bound),
                       b3 = __ballot_sync(kFullMask, t.w >= bound);
        const int all = (__popc(b0) + __popc(b1)) + (__popc(b2) + __popc(b3));
        if (all == 0) continue;
        uint32_t at = (uint32_t)(kept + (__popc(b0 & below) + __popc(b1 & below)) + (__popc(b2 & below) + __popc(b3 & below)));
        kept += all;
        if (kept > p.tokens_cap) break;
        __syncwarp();                                      // these 128 have been read by all lanes: the list may come over them
        const int token = 4 * (32 * i + lane);
        take(t.x, at, token); take(t.y, at, token + 1); take(t.z, at, token + 2); take(t.w, at, token + 3);
      }
      __syncwarp();
      if (kept <= p.tokens_cap) {
        const RowShared list{vals, tokens, kept};
        limit_and_draw<NW, BF16>(p, list, tm, sh, r, m, l, sc, whole_row, LeftOut<BF16>{row, bound}, row.inf);
        return;
      }
      for (int i = 0; i < iters; ++i) shared[first + 32 * i] = first + 32 * i < quads ? row.quad(first + 32 * i) : none();
    } else {
    // Four quads at a time: counts in the bytes of a word, summed over the lanes at once.
    static_assert(kSampleMostV <= 4 * 32 * 32 * 16, "");   // at most 16 quads a thread
    uint32_t counts[4] = {0, 0, 0, 0};
    int mine = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (4 * g >= iters) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 t = 4 * g + i < iters ? quad(first + 32 * (4 * g + i)) : none();
        counts[g] += ((uint32_t)(t.x >= bound) + (uint32_t)(t.y >= bound) + (uint32_t)(t.z >= bound) + (uint32_t)(t.w >= bound)) << (8 * i);
      }
      mine += (int)((counts[g] * 0x01010101u) >> 24);      // the four bytes' sum: at most 16
    }
    int before = 0, kept;                                  // elements of the list in front of this warp's, and in all
    if (NW == 1) {
      kept = __reduce_add_sync(kFullMask, mine);
    } else {
      const int upto = tm.scan(mine);
      int* starts = reinterpret_cast<int*>(sh.hist);       // (free by now)
      tm.sync();
      if (lane == 31) starts[warp] = upto;
      tm.sync();
      before = warp > 0 ? starts[warp - 1] : 0;
      kept = starts[NW - 1];
    }
    if (kept <= p.tokens_cap) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (4 * g >= iters) break;
        uint32_t upto = counts[g];                         // at most 128 a byte
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(kFullMask, upto, o);
          if (lane >= o) upto += v;
        }
        const uint32_t all = __shfl_sync(kFullMask, upto, 31), own = upto - counts[g];
        float4 t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = 4 * g + i < iters ? quad(first + 32 * (4 * g + i)) : none();
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          int at = before + (int)((own >> (8 * i)) & 255u);
          const int token = 4 * (first + 32 * (4 * g + i));
          auto take = [&](float x, int j) {
            if (x >= bound) { vals[at] = x; tokens[at] = (uint16_t)(token + j); ++at; }
          };
          take(t[i].x, 0); take(t[i].y, 1); take(t[i].z, 2); take(t[i].w, 3);
          before += (int)((all >> (8 * i)) & 255u);
        }
        __syncwarp();
      }
      tm.sync();
      const RowShared list{vals, tokens, kept};
      limit_and_draw<NW, BF16>(p, list, tm, sh, r, m, l, sc, whole_row, LeftOut<BF16>{row, bound}, row.inf);
      return;
    }
    }
  }
  // no limit, or one that leaves more than a list takes: the whole row
  if constexpr (WHOLE) {
    if (!SHARED) {
      for (int i = 0; i < iters; ++i)
        if (first + 32 * i < quads) shared[first + 32 * i] = quad(first + 32 * i);
    }
    tm.sync();
    const RowShared all{vals, nullptr, p.V};
    limit_and_draw<NW, BF16>(p, all, tm, sh, r, m, l, sc, Sum<NW>(0), LeftOut<BF16>{row, 0.f}, row.inf);
  } else {
    limit_and_draw<NW, BF16>(p, row, tm, sh, r, m, l, sc, Sum<NW>(0), LeftOut<BF16>{row, 0.f}, row.inf);
  }
}

// LISTS: with allow bits.
template <int NW, bool BF16, bool LISTS, bool SHARED>
__global__ void __launch_bounds__(NW == 1 ? 64 : NW * 32, NW == 1 ? 16 : (NW == 32 ? 1 : 24 / NW))
sample_kernel(const SampleParams p) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int NT = NW * 32, kTeams = NW == 1 ? 2 : 1;
  const int team = NW == 1 ? threadIdx.x >> 5 : 0;
  const int64_t r = (int64_t)blockIdx.x * kTeams + team;
  if (r >= p.R) return;                                    // whole teams
  SampleShared<NW>& sh = *reinterpret_cast<SampleShared<NW>*>(smem + (size_t)team * p.team_bytes);
  float* vals = reinterpret_cast<float*>(&sh + 1);
  uint16_t* tokens = reinterpret_cast<uint16_t*>(vals + p.cap);
  static_assert(sizeof(SampleShared<NW>) % 16 == 0, "");
  const Team<NW> tm{NW == 1 ? (int)(threadIdx.x & 31) : (int)threadIdx.x, sh.red};
  RowLimits l = row_limits(p, r, tm.tid);
  const int words = (p.V + 63) >> 6;
  const uint64_t* allow = LISTS ? p.allow + r * words : nullptr;
  const RowGlobal<BF16> row{reinterpret_cast<const char*>(p.logits) + r * p.ld * (BF16 ? 2 : 4), allow, p.V, p.vec, false};
  int n = p.V;
  if constexpr (LISTS) {
    // the allowed tokens' places: a thread has a word (run_sample's rows have no more words than threads)
    uint64_t a = tm.tid < words ? __ldg(allow + tm.tid) : 0ull;
    if (tm.tid == words - 1 && (p.V & 63)) a &= (1ull << (p.V & 63)) - 1ull;
    const int count = __popcll(a), upto = tm.scan(count);
    n = NW == 1 ? __shfl_sync(kFullMask, upto, 31) : tm.reduce(upto, [](int a, int b) { return max(a, b); });
    if (n <= p.tokens_cap) {
      int at = upto - count;
      const int token0 = tm.tid * 64;
      for (uint32_t h = (uint32_t)a; h != 0u; h &= h - 1u) tokens[at++] = (uint16_t)(token0 + __ffs((int)h) - 1);
      for (uint32_t h = (uint32_t)(a >> 32); h != 0u; h &= h - 1u) tokens[at++] = (uint16_t)(token0 + 31 + __ffs((int)h));
      tm.sync();
      float m = -INFINITY;
      for (int i0 = 0; i0 < n; i0 += 4 * NT) {             // four loads in flight
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = i0 + i * NT + tm.tid;
          x[i] = j < n ? logit_at<BF16>(row.row, tokens[j]) : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = i0 + i * NT + tm.tid;
          if (j < n) vals[j] = x[i];
          m = max_nan(m, x[i]);
        }
      }
      m = tm.reduce(m, [](float a, float b) { return max_nan(a, b); });
      tm.sync();
      if (!(m > -INFINITY)) {                              // nothing, or NaN
        if (m != m && tm.tid == 0) flag_status(p.d_status, GRACE_DEV_NAN);
        store_all<NW>(p, l, tm, r, 0, 0.f, -INFINITY);
        return;
      }
      const bool infinite = m == INFINITY;
      if (infinite) {                                      // those at +inf weigh 1 each, all others nothing
        for (int i = tm.tid; i < n; i += NT) vals[i] = vals[i] == INFINITY ? 0.f : -INFINITY;
        tm.sync();
        m = 0.f;
      }
      if (!(l.temperature > 0.f)) {
        int first = 0x7fffffff;
        for (int i = tm.tid; i < n; i += NT)
          if (vals[i] == m) first = min(first, i);
        first = tm.reduce(first, [](int a, int b) { return min(a, b); });
        store_all<NW>(p, l, tm, r, tokens[first], infinite ? INFINITY : m, 0.f);
        return;
      }
      const RowShared list{vals, tokens, n};
      const Scale sc(l.temperature);
      if (l.min_p > 0.f) l.least = min_p_bound(m, l.min_p, sc.t);
      limit_and_draw<NW, BF16>(p, list, tm, sh, r, m, l, sc, Sum<NW>(0), LeftOut<BF16>{row, 0.f}, infinite);
      return;
    }
  }
  sample_dense<NW, BF16, SHARED, !LISTS && NW != 32>(p, row, tm, sh, vals, tokens, r, n, l);
}

template <int NW, bool BF16, bool LISTS>
static grace_status_t launch_sample(SampleParams p, cudaStream_t s) {
  // Without a constraint a warp's row lies in shared memory from the start (SHARED); a longer one of up to 16384 tokens, read by
  // every pass before, comes there when no list of half its tokens holds what can be kept.  Under a constraint there is room
  // for half the tokens; a row with more allowed ones is read by every pass, as are longer rows.
  constexpr bool kShared = NW == 1 && !LISTS;
  constexpr int kTeams = NW == 1 ? 2 : 1;
  const int row = kShared ? (p.V + 127) & ~127 : (p.V + 15) & ~15, half = p.V <= 512 ? row : (p.V / 2 + 15) & ~15;
  p.cap = NW == 32 ? 16384 : (LISTS ? half : row);         // (V <= 2048, 8192, 16384 with 1, 4, 8 warps: sample_dense's WHOLE)
  static_assert(kSampleMostV <= 32 * 32 * 64, "");         // 64 tokens a thread
  p.tokens_cap = NW == 32 ? 16384 : half;
  p.team_bytes = ((int)sizeof(SampleShared<NW>) + p.cap * 4 + p.tokens_cap * 2 + 15) & ~15;
  static_assert(sizeof(SampleShared<32>) + 16384 * 6 <= 227 * 1024, "");
  static unsigned long long attr_set_devices = 0;
  DeviceSetup su(&attr_set_devices);
  if (su) {
    GRACE_CUDA_TRY(cudaFuncSetAttribute(sample_kernel<NW, BF16, LISTS, kShared>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
    su.done();
  }
  GRACE_CUDA_TRY(launch_pdl(sample_kernel<NW, BF16, LISTS, kShared>, dim3((unsigned)((p.R + kTeams - 1) / kTeams)), dim3(NW == 1 ? 64 : NW * 32),
                            (size_t)p.team_bytes * kTeams, s, p));
  GRACE_LAUNCH_CHECK();
  return GRACE_OK;
}
template <bool BF16>
static grace_status_t run_sample(const SampleParams& p, cudaStream_t s) {
  // Warps of a row: one per 2048 tokens at least, more while the GPU is not filled by the rows (a pass over a row is then as
  // long as its threads' part).
  // Rows in a list's shared memory: half the tokens' room.  (With 3/8 of it 20 warps instead of 18 are on an SM, 8 % less time for short
  // lists, but top-k 1000 of 2048 goes from 517 to 670 us, its row being read again.)
  const bool lists = p.allow != nullptr;
  // (64 tokens a thread at the most: sample_kernel's words)
  if (p.V > 16384) return lists ? launch_sample<32, BF16, true>(p, s) : launch_sample<32, BF16, false>(p, s);
  if (p.V > 8192 || (p.V > 1024 && p.R <= kSms)) return lists ? launch_sample<8, BF16, true>(p, s) : launch_sample<8, BF16, false>(p, s);
  if (p.V > 2048 || (p.V > 256 && p.R <= 4 * kSms)) return lists ? launch_sample<4, BF16, true>(p, s) : launch_sample<4, BF16, false>(p, s);
  return lists ? launch_sample<1, BF16, true>(p, s) : launch_sample<1, BF16, false>(p, s);
}

}  // namespace grace
