// Tokens drawn from a row's (allowed) logits: temperature, top-k, top-p, min-p, one uniform number per draw.
//
//   w_v = e^((x_v - max) / T) over the allowed tokens, in the order (x descending, token ascending).  Every limit leaves a
//   prefix of that order, so what is kept is a cut (t, i): tokens with x > t, and of those with x = t the ones up to token i.
//   A draw takes the first kept token, in ascending order, at which the running sum of kept weights exceeds u times the whole.
//
// No sort: the cut is found through a histogram of 256 equal steps of (max - x) / T, in counts (top-k) or in fixed-point
// weights (top-p), whose one bucket that holds the cut is then resolved value by value.
// The answer is that of the definition in 64 bits, at the cost of 32: weights and sums are fp32, every comparison of a sum with
// a border has a margin above the sums' worst error, and a row for which one falls inside the margin is done again with
// e^ and sums in fp64.
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
  int M, V, draws, vec;          // vec: rows start on 16 bytes
  int list_cap;                  // elements of the row buffer
};

constexpr int kSampleBuckets = 256;
// Steps of the histogram: 256 over 22 powers of two of weight; the last one holds all that is lighter.
constexpr float kSampleSteps = 256.f / 22.f;
constexpr int kSampleMostV = 65536;

__device__ __forceinline__ float sample_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

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

// A row's elements by place: place = order of the tokens.  Places beyond the last hold -inf.
struct RowShared {               // in shared memory: a whole row, or the allowed elements of one with their tokens
  const float* vals;
  const uint16_t* tokens;        // NULL: token = place
  int n;
  __device__ __forceinline__ int quads() const { return (n + 3) >> 2; }
  __device__ __forceinline__ float4 quad(int q) const { return reinterpret_cast<const float4*>(vals)[q]; }
  __device__ __forceinline__ int token(int place) const { return tokens != nullptr ? tokens[place] : place; }
};
template <bool BF16>
struct RowGlobal {               // read again by every pass (out of L2): a row longer than the buffer
  const char* row;
  const uint64_t* allow;
  int n, vec;
  bool inf;                      // the row's largest is +inf: these weigh 1, all others nothing
  __device__ __forceinline__ int quads() const { return (n + 3) >> 2; }
  __device__ __forceinline__ float4 quad(int q) const {
    const int at = q << 2;
    uint32_t bits = allow != nullptr ? (uint32_t)(__ldg(allow + (at >> 6)) >> (at & 63)) & 15u : 15u;
    if (at + 4 > n) bits &= (1u << (n - at)) - 1u;
    float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (bits != 0u) {
      if (vec && at + 4 <= n) {
        if (BF16) {
          const uint2 t = __ldg(reinterpret_cast<const uint2*>(row) + q);
          v[0] = bf16_lo(t.x); v[1] = bf16_hi(t.x); v[2] = bf16_lo(t.y); v[3] = bf16_hi(t.y);
        } else {
          const float4 t = __ldg(reinterpret_cast<const float4*>(row) + q);
          v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((bits >> j) & 1u)
            v[j] = BF16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(row) + at + j) << 16)
                        : __ldg(reinterpret_cast<const float*>(row) + at + j);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!((bits >> j) & 1u)) v[j] = -INFINITY;
      if (inf) v[j] = v[j] == INFINITY ? 0.f : -INFINITY;
    }
    return make_float4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ int token(int place) const { return place; }
};

struct Cut {
  float t;                       // x > t, or x = t and place <= last
  int last;
  __device__ __forceinline__ bool keeps(float x, int place) const { return x > t || (x == t && place <= last); }
};

// A team's shared memory besides the row.
template <int NW>
struct SampleShared {
  static constexpr int kList = NW == 1 ? 64 : 256;
  uint32_t hist[kSampleBuckets];
  float list[kList];
  double prefix[NW * 32];
  double red[NW < 2 ? 2 : NW];
  int n_list, bucket, found, found_r, found_all;
  uint32_t above;
  float found_t;
};

template <class F>
__device__ __forceinline__ void each(float4 v, F f) { f(v.x, 0); f(v.y, 1); f(v.z, 2); f(v.w, 3); }

template <int NW, class Row>
struct Sampler {
  const Row& row;
  const Team<NW>& tm;
  SampleShared<NW>& sh;
  float m;                       // largest value
  float c;                       // log2(e) / T
  double inv_t;                  // 1 / T
  float margin;                  // of sums, relative to the whole
  static constexpr int NT = NW * 32;

  __device__ __forceinline__ float weight(float x) const { return sample_ex2((x - m) * c); }
  __device__ __forceinline__ double weight64(float x) const { return exp(((double)x - (double)m) * inv_t); }
  __device__ __forceinline__ int bucket_of(float x) const { return min(kSampleBuckets - 1, (int)((m - x) * c * kSampleSteps)); }

  template <class F>
  __device__ __forceinline__ void for_each(F f) const {
    for (int q = tm.tid; q < row.quads(); q += NT) {
      const float4 v = row.quad(q);
      each(v, [&](float x, int j) { f(x, 4 * q + j); });
    }
  }

  // First bucket at which the histogram's running sum reaches `target` (sh.bucket) and the sum in front of it (sh.above);
  // -1 if none does.
  __device__ __forceinline__ void find_bucket(uint32_t target) const {
    if (tm.tid < 32) {
      const int lane = tm.tid;
      uint32_t h[8], s = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) { h[j] = sh.hist[8 * lane + j]; s += h[j]; }
      uint32_t incl = s;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(kFullMask, incl, o);
        if (lane >= o) incl += t;
      }
      const uint32_t reached = __ballot_sync(kFullMask, incl >= target);
      if (reached == 0u) {
        if (lane == 0) sh.bucket = -1;
      } else if (lane == __ffs(reached) - 1) {
        uint32_t run = incl - s;
        bool open = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (open && run + h[j] >= target) { sh.bucket = 8 * lane + j; sh.above = run; open = false; }
          run += h[j];
        }
      }
    }
    tm.sync();
  }

  // Narrows `cut` to its first k elements (MASS false), or to the fewest whose weights reach p of the sum of its weights.
  template <bool MASS>
  __device__ __noinline__ Cut narrow(const Cut cut, const int k, const float p) const {
    const float scale = MASS ? exp2f(31.f - ceilf(log2f((float)(4 * row.quads())))) : 1.f;   // fixed point: any row's sum below 2^32
    auto share = [&](float x) { return MASS ? __float2uint_rn(weight(x) * scale) : 1u; };
    for (int i = tm.tid; i < kSampleBuckets; i += NT) sh.hist[i] = 0u;
    if (tm.tid == 0) { sh.n_list = 0; sh.found = 0; }
    tm.sync();
    for_each([&](float x, int place) {
      if (cut.keeps(x, place)) atomicAdd(&sh.hist[bucket_of(x)], share(x));
    });
    tm.sync();
    uint32_t goal = (uint32_t)k;
    if (MASS) {
      uint32_t all = 0;
      for (int i = tm.tid; i < kSampleBuckets; i += NT) all += sh.hist[i];
      all = tm.sum(all);
      goal = max(1u, (uint32_t)fminf((float)all * p, 4294967040.f));
      goal = min(goal, all);
    }
    find_bucket(goal);
    if (sh.bucket < 0) return cut;                         // no more than k elements
    const int b = sh.bucket;
    float whole = 0.f, above = 0.f;
    int n_above = (int)sh.above;
    for_each([&](float x, int place) {
      if (!cut.keeps(x, place)) return;
      const int at = bucket_of(x);
      if (MASS) {
        const float w = weight(x);
        whole += w;
        if (at < b) above += w;
      }
      if (at == b) {
        const int i = atomicAdd(&sh.n_list, 1);
        if (i < sh.kList) sh.list[i] = x;
      }
    });
    if (MASS) { whole = tm.sum(whole); above = tm.sum(above); }
    tm.sync();
    int n = sh.n_list;
    // the bracket by value; only needed beyond the list, but for 64 bits too
    uint32_t key_lo = 0xffffffffu, key_hi = 0u;
    if (n <= sh.kList) {
      for (int i = tm.tid; i < n; i += NT) { const uint32_t key = ordered_key(sh.list[i]); key_lo = min(key_lo, key); key_hi = max(key_hi, key); }
    } else {
      for_each([&](float x, int place) {
        if (cut.keeps(x, place) && bucket_of(x) == b) { const uint32_t key = ordered_key(x); key_lo = min(key_lo, key); key_hi = max(key_hi, key); }
      });
    }
    key_lo = tm.reduce(key_lo, [](uint32_t a, uint32_t d) { return min(a, d); });
    key_hi = tm.reduce(key_hi, [](uint32_t a, uint32_t d) { return max(a, d); });
    if (n > sh.kList) {
      // more values than the list takes: histograms of equal steps of the ordered bits, until they fit or are all the same
      while (n > sh.kList && key_lo < key_hi) {
        const uint32_t range = key_hi - key_lo;
        const int shift = max(0, 24 - __clz(range));
        tm.sync();
        for (int i = tm.tid; i < kSampleBuckets; i += NT) sh.hist[i] = 0u;
        tm.sync();
        for_each([&](float x, int place) {
          const uint32_t key = ordered_key(x);
          if (key >= key_lo && key <= key_hi && cut.keeps(x, place)) atomicAdd(&sh.hist[(key_hi - key) >> shift], share(x));
        });
        tm.sync();
        uint32_t want = (uint32_t)(k - n_above);
        if (MASS) {
          uint32_t all = 0;
          for (int i = tm.tid; i < kSampleBuckets; i += NT) all += sh.hist[i];
          all = tm.sum(all);
          want = min(max(1u, (uint32_t)fminf(fmaxf((p * whole - above) * scale, 1.f), 4294967040.f)), max(1u, all));
        }
        find_bucket(want);
        const int at = max(0, sh.bucket);
        key_hi -= (uint32_t)at << shift;
        key_lo = max(key_lo, key_hi - ((1u << shift) - 1u));
        float more = 0.f;
        int inside = 0, over = 0;
        for_each([&](float x, int place) {
          if (!cut.keeps(x, place)) return;
          const uint32_t key = ordered_key(x);
          if (key > key_hi) { over += 1; if (MASS) more += weight(x); }
          else if (key >= key_lo) inside += 1;
        });
        n = tm.sum(inside);
        n_above = tm.sum(over);
        if (MASS) above = tm.sum(more);
      }
      tm.sync();
      if (tm.tid == 0) sh.n_list = 0;
      tm.sync();
      if (key_lo < key_hi) {
        for_each([&](float x, int place) {
          const uint32_t key = ordered_key(x);
          if (key >= key_lo && key <= key_hi && cut.keeps(x, place)) { const int i = atomicAdd(&sh.n_list, 1); if (i < sh.kList) sh.list[i] = x; }
        });
      } else {
        for_each([&](float x, int place) {                 // one value, many times
          if (ordered_key(x) == key_hi && cut.keeps(x, place)) sh.list[0] = x;
        });
      }
      tm.sync();
    }
    const int copies = key_lo == key_hi ? n : 1;           // of every list entry
    const int len = key_lo == key_hi ? min(n, 1) : n;
    // The list resolved: the value at which the count or the sum of weights in front passes the goal.
    for (int i = tm.tid; i < len; i += NT) {
      const float x = sh.list[i];
      int same = 0;
      if (MASS) {
        float front = above;
        for (int j = 0; j < len; ++j) {
          const float y = sh.list[j];
          if (y > x) front += weight(y);
          same += y == x;
        }
        same *= copies;
        const float w = weight(x), gap = p * whole - front, slack = margin * whole;
        if (gap > slack && gap + slack < w * (float)same) {
          const float q = gap / w, r = ceilf(q);
          if (same == 1 || ((r - q) * w > slack && (q - (r - 1.f)) * w > slack)) {
            sh.found_t = x; sh.found_r = min(same, max(1, (int)r)); sh.found_all = sh.found_r == same; sh.found = 1;
          }
        }
      } else {
        int front = n_above;
        for (int j = 0; j < len; ++j) { const float y = sh.list[j]; front += y > x; same += y == x; }
        same *= copies;
        if (front < k && k <= front + same) { sh.found_t = x; sh.found_r = k - front; sh.found_all = sh.found_r == same; sh.found = 1; }
      }
    }
    tm.sync();
    if (MASS && sh.found == 0) narrow64(cut, p, key_lo, key_hi, len, copies);
    Cut out = {sh.found_t, 0x7fffffff};
    if (sh.found_all != 0) {
      if (out.t == cut.t) out.last = cut.last;
      return out;
    }
    // some of the ties only: the found_r-th of them by place
    const int r = sh.found_r;
    int lo = 0, hi = 4 * row.quads() - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      int up_to = 0;
      for_each([&](float x, int place) { up_to += x == out.t && place <= mid && cut.keeps(x, place); });
      if (tm.sum(up_to) >= r) hi = mid; else lo = mid + 1;
    }
    out.last = lo;
    return out;
  }

  // The same decision by sums in 64 bits: first within the bracket that 32 bits found, then, should the border lie outside it,
  // by bisection over all values.  Sets sh.found_*.
  __device__ __noinline__ void narrow64(const Cut cut, const float p, const uint32_t key_lo, const uint32_t key_hi, const int len, const int copies) const {
    double whole = 0., above = 0.;
    for_each([&](float x, int place) {
      if (!cut.keeps(x, place)) return;
      const double w = weight64(x);
      whole += w;
      if (ordered_key(x) > key_hi) above += w;
    });
    whole = tm.sum(whole);
    above = tm.sum(above);
    const double goal = (double)p * whole;
    auto settle = [&](float x, double front, int same) {
      const double w = weight64(x);
      const int r = min(same, max(1, (int)fmin(ceil((goal - front) / w), 2147483647.)));
      sh.found_t = x; sh.found_r = r; sh.found_all = r == same; sh.found = 1;
    };
    for (int i = tm.tid; i < len; i += NT) {
      const float x = sh.list[i];
      double front = above;
      int same = 0;
      for (int j = 0; j < len; ++j) {
        const float y = sh.list[j];
        if (y > x) front += weight64(y);
        same += y == x;
      }
      same *= copies;
      if ((front < goal || (front == 0. && goal <= 0.)) && front + weight64(x) * same >= goal) settle(x, front, same);
    }
    tm.sync();
    if (sh.found != 0) return;
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
      else { sh.found_t = least; sh.found_r = 1; sh.found_all = 1; sh.found = 1; }
    }
    tm.sync();
  }

  // Sums of the kept weights by quads (table) and by the threads' ranges of them (sh.prefix, inclusive); returns the whole.
  template <class F>
  __device__ __forceinline__ F build(const Cut cut, F* table) const {
    tm.sync();
    for (int q = tm.tid; q < row.quads(); q += NT) {
      const float4 v = row.quad(q);
      F s = F(0);
      each(v, [&](float x, int j) { if (cut.keeps(x, 4 * q + j)) s += sizeof(F) == 8 ? (F)weight64(x) : (F)weight(x); });
      table[q] = s;
    }
    tm.sync();
    const int per = (row.quads() + NT - 1) / NT;
    F s = F(0);
    for (int i = 0; i < per; ++i) {
      const int q = tm.tid * per + i;
      if (q < row.quads()) s += table[q];
    }
    s = tm.scan(s);
    F* prefix = reinterpret_cast<F*>(sh.prefix);
    prefix[tm.tid] = s;
    tm.sync();
    return prefix[NT - 1];
  }

  // Place of the first kept element at which the running sum exceeds u * whole; `sure` unless a border is within `slack`.
  template <class F>
  __device__ __forceinline__ int pick(const Cut cut, const F* table, F whole, float u, F slack, bool& sure) const {
    const F* prefix = reinterpret_cast<const F*>(sh.prefix);
    const F goal = (F)u * whole;
    const int per = (row.quads() + NT - 1) / NT;
    int lo = 0, hi = NT - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (prefix[mid] > goal) hi = mid; else lo = mid + 1;
    }
    F run = lo > 0 ? prefix[lo - 1] : F(0);
    int place = -1, last = -1;
    sure = false;
    // the threads' ranges in turn: rounding may leave the border just behind the first one
    for (int q = lo * per; q < row.quads() && place < 0; ++q) {
      const F s = table[q];
      if (run + s > goal || q + 1 == row.quads()) {
        const float4 v = row.quad(q);
        each(v, [&](float x, int j) {
          const F w = cut.keeps(x, 4 * q + j) ? (sizeof(F) == 8 ? (F)weight64(x) : (F)weight(x)) : F(0);
          if (place < 0 && w > F(0)) {
            last = 4 * q + j;
            if (run + w > goal) { place = last; sure = goal - run > slack && run + w - goal > slack; }
          }
          run += w;
        });
      } else {
        run += s;
      }
    }
    if (place < 0) {
      // u next to 1: the last kept element with a weight
      place = last;
      for (int q = row.quads() - 1; q >= 0 && place < 0; --q) {
        const float4 v = row.quad(q);
        each(v, [&](float x, int j) {
          const F w = cut.keeps(x, 4 * q + j) ? (sizeof(F) == 8 ? (F)weight64(x) : (F)weight(x)) : F(0);
          if (w > F(0)) place = 4 * q + j;
        });
      }
    }
    return place;
  }
};

__device__ __forceinline__ float sample_logit(const SampleParams& p, bool bf16, int64_t r, int token) {
  return bf16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p.logits) + r * p.ld + token) << 16)
              : __ldg(reinterpret_cast<const float*>(p.logits) + r * p.ld + token);
}

// All draws of a row whose elements `row` holds.
template <int NW, bool BF16, class Row>
__device__ __forceinline__ void sample_row(const SampleParams& p, Row& row, const Team<NW>& tm, SampleShared<NW>& sh, void* table, int64_t r,
                                           float m, bool nan, bool infinite) {
  constexpr int NT = NW * 32;
  const int b = (int)(r / p.M), beam = (int)(r % p.M);
  float* out_score = p.out_score + r * p.draws;
  float* out_logq = p.out_logq != nullptr ? p.out_logq + r * p.draws : nullptr;
  int32_t* out_token = p.out_token + r * p.draws;
  int32_t* out_parent = p.out_parent != nullptr ? p.out_parent + r * p.draws : nullptr;
  const float base = p.row_score != nullptr ? __ldg(p.row_score + r) : 0.f, lse = p.row_lse != nullptr ? __ldg(p.row_lse + r) : 0.f;
  auto store = [&](int d, int token, float logq) {
    out_token[d] = token;
    if (out_parent != nullptr) out_parent[d] = beam;
    out_score[d] = logq == -INFINITY ? -INFINITY : base + (sample_logit(p, BF16, r, token) - lse);
    if (out_logq != nullptr) out_logq[d] = logq;
  };
  if (nan || m == -INFINITY) {
    if (nan && tm.tid == 0) flag_status(p.d_status, GRACE_DEV_NAN);
    for (int d = tm.tid; d < p.draws; d += NT) store(d, 0, -INFINITY);
    return;
  }
  if (infinite) m = 0.f;
  const float temperature = p.temperature != nullptr ? __ldg(p.temperature + b) : 1.f;
  Sampler<NW, Row> s{row, tm, sh, m, 0.f, 0., row.quads() > 512 ? 0x1p-17f : 0x1p-18f};
  if (!(temperature > 0.f)) {
    int first = 0x7fffffff;
    s.for_each([&](float x, int place) { if (x == m) first = min(first, place); });
    first = tm.reduce(first, [](int a, int d) { return min(a, d); });
    const int token = row.token(first);
    for (int d = tm.tid; d < p.draws; d += NT) store(d, token, 0.f);
    return;
  }
  const double t64 = fmin((double)temperature, 1e30);
  s.inv_t = 1. / t64;
  s.c = (float)fmin(1.4426950408889634 * s.inv_t, 1e38);
  Cut cut = {-INFINITY, -1};
  const int k = p.top_k != nullptr ? __ldg(p.top_k + b) : 0;
  if (k > 0 && k < row.n) cut = s.template narrow<false>(cut, k, 0.f);
  const float top_p = p.top_p != nullptr ? __ldg(p.top_p + b) : 1.f;
  if (top_p < 1.f) {
    tm.sync();
    cut = s.template narrow<true>(cut, 0, fmaxf(top_p, 0.f));
  }
  const float min_p = p.min_p != nullptr ? __ldg(p.min_p + b) : 0.f;
  if (min_p > 0.f) {
    // w >= min_p as a bound on x, rounded up to the next fp32
    const float least = min_p < 1.f ? fminf(m, __double2float_ru((double)m + t64 * log((double)min_p))) : m;
    if (least > cut.t) cut = Cut{least, 0x7fffffff};
  }
  float* table32 = reinterpret_cast<float*>(table);
  double* table64 = reinterpret_cast<double*>(table);
  const float whole = s.template build<float>(cut, table32);
  const float log_whole = logf(whole);
  bool have64 = false;
  double whole64 = 0.;
  for (int d0 = 0; d0 < p.draws; d0 += NT) {
    const int d = d0 + tm.tid;
    const bool in = d < p.draws;
    float u = in ? __ldg(p.u + r * p.draws + d) : 0.5f;
    u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    bool sure = false;
    int place = -1;
    if (!have64 && in) place = s.template pick<float>(cut, table32, whole, u, s.margin * whole, sure);
    const int doubt = tm.reduce(in && !sure ? 1 : 0, [](int a, int e) { return a | e; });
    if (doubt) {
      if (!have64) { whole64 = s.template build<double>(cut, table64); have64 = true; }
      bool ignored;
      if (in && !sure) place = s.template pick<double>(cut, table64, whole64, u, 0., ignored);
    }
    if (in) {
      const int token = row.token(max(place, 0));
      const float x = infinite ? 0.f : sample_logit(p, BF16, r, token);
      store(d, token, (float)(((double)x - (double)m) * s.inv_t) - log_whole);
    }
  }
}

template <int NW, bool BF16>
__global__ void __launch_bounds__(NW == 1 ? 128 : NW * 32)
sample_kernel(const SampleParams p, const int shared_row) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int NT = NW * 32, kTeams = NW == 1 ? 4 : 1;
  const int team = NW == 1 ? threadIdx.x >> 5 : 0;
  const int64_t r = (int64_t)blockIdx.x * kTeams + team;
  if (r >= p.R) return;                                    // whole teams
  uint8_t* mine = smem + (size_t)team * shared_row;
  SampleShared<NW>& sh = *reinterpret_cast<SampleShared<NW>*>(mine);
  void* table = mine + ((sizeof(SampleShared<NW>) + 15) & ~(size_t)15);
  const int quads = (p.V + 3) >> 2;
  float* vals = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(table) + (((size_t)quads * 8 + 15) & ~(size_t)15));
  uint16_t* tokens = reinterpret_cast<uint16_t*>(vals + p.list_cap);
  const Team<NW> tm{NW == 1 ? (int)(threadIdx.x & 31) : (int)threadIdx.x, sh.red};
  const char* logits = reinterpret_cast<const char*>(p.logits) + r * p.ld * (BF16 ? 2 : 4);
  const int words = (p.V + 63) >> 6;
  const uint64_t* allow = p.allow != nullptr ? p.allow + r * words : nullptr;
  auto load = [&](int token) {
    return BF16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(logits) + token) << 16) : __ldg(reinterpret_cast<const float*>(logits) + token);
  };
  float m = -INFINITY;
  int nan = 0;
  auto see = [&](float x) { m = fmaxf(m, x); nan |= x != x; };
  auto most = [](float a, float b) { return fmaxf(a, b); };
  auto either = [](int a, int b) { return a | b; };

  int n = p.V;                                             // elements of the row buffer
  if (allow != nullptr) {
    // the allowed tokens' places: a thread's words are neighbours, so that the list is in order
    const int per = (words + NT - 1) / NT;
    auto word = [&](int i) {
      const int w = tm.tid * per + i;
      uint64_t a = w < words ? __ldg(allow + w) : 0ull;
      if (w == words - 1 && (p.V & 63)) a &= (1ull << (p.V & 63)) - 1ull;
      return a;
    };
    int count = 0;
    for (int i = 0; i < per; ++i) count += __popcll(word(i));
    const int upto = tm.scan(count);
    n = tm.reduce(upto, [](int a, int b) { return max(a, b); });
    if (n <= p.list_cap) {
      int at = upto - count;
      for (int i = 0; i < per; ++i) {
        uint64_t a = word(i);
        while (a != 0ull) {
          const int bit = __ffsll((long long)a) - 1;
          a &= a - 1ull;
          tokens[at++] = (uint16_t)((tm.tid * per + i) * 64 + bit);
        }
      }
      tm.sync();
      for (int i = tm.tid; i < n; i += NT) { const float x = load(tokens[i]); vals[i] = x; see(x); }
    }
  } else if (n <= p.list_cap) {
    if (p.vec) {
      for (int q = tm.tid; q < (n >> 2); q += NT) {
        float4 t;
        if (BF16) {
          const uint2 w = __ldg(reinterpret_cast<const uint2*>(logits) + q);
          t = make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
        } else {
          t = __ldg(reinterpret_cast<const float4*>(logits) + q);
        }
        reinterpret_cast<float4*>(vals)[q] = t;
        see(t.x); see(t.y); see(t.z); see(t.w);
      }
      for (int i = (n & ~3) + tm.tid; i < n; i += NT) { const float x = load(i); vals[i] = x; see(x); }
    } else {
      for (int i = tm.tid; i < n; i += NT) { const float x = load(i); vals[i] = x; see(x); }
    }
  }
  if (n <= p.list_cap) {
    for (int i = n + tm.tid; i < ((n + 3) & ~3); i += NT) vals[i] = -INFINITY;
    m = tm.reduce(m, most);
    nan = tm.reduce(nan, either);
    tm.sync();
    if (m == INFINITY) {                                   // those at +inf weigh 1 each, all others nothing
      for (int i = tm.tid; i < n; i += NT) vals[i] = vals[i] == INFINITY ? 0.f : -INFINITY;
      tm.sync();
    }
    RowShared row{vals, allow != nullptr ? tokens : nullptr, n};
    sample_row<NW, BF16>(p, row, tm, sh, table, r, m, nan != 0, m == INFINITY);
  } else if constexpr (NW == 32) {
    RowGlobal<BF16> row{logits, allow, p.V, p.vec, false};
    for (int q = tm.tid; q < row.quads(); q += NT) { const float4 t = row.quad(q); see(t.x); see(t.y); see(t.z); see(t.w); }
    m = tm.reduce(m, most);
    nan = tm.reduce(nan, either);
    row.inf = m == INFINITY;
    sample_row<NW, BF16>(p, row, tm, sh, table, r, m, nan != 0, m == INFINITY);
  }
}

// Shared memory of a team: its struct, the table of quad sums (fp64 where it comes to that), the row buffer.
template <int NW>
static int sample_shared_bytes(int V, int list_cap, bool lists) {
  const int quads = (V + 3) >> 2;
  int n = (int)((sizeof(SampleShared<NW>) + 15) & ~(size_t)15) + ((quads * 8 + 15) & ~15) + list_cap * 4;
  if (lists) n += (list_cap * 2 + 15) & ~15;
  return (n + 15) & ~15;
}

template <int NW, bool BF16>
static grace_status_t launch_sample(SampleParams p, int list_cap, cudaStream_t s) {
  p.list_cap = list_cap;
  const int one = sample_shared_bytes<NW>(p.V, list_cap, p.allow != nullptr), teams = NW == 1 ? 4 : 1;
  static unsigned long long attr_set_devices = 0;
  DeviceSetup su(&attr_set_devices);
  if (su) {
    GRACE_CUDA_TRY(cudaFuncSetAttribute(sample_kernel<NW, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
    su.done();
  }
  GRACE_CUDA_TRY(launch_pdl(sample_kernel<NW, BF16>, dim3((unsigned)((p.R + teams - 1) / teams)), dim3(NW == 1 ? 128 : NW * 32), (size_t)one * teams, s, p, one));
  GRACE_LAUNCH_CHECK();
  return GRACE_OK;
}
template <bool BF16>
static grace_status_t run_sample(const SampleParams& p, cudaStream_t s) {
  const int row = (p.V + 15) & ~15;
  if (p.V <= 2048) return launch_sample<1, BF16>(p, row, s);
  if (p.V <= 12288) return launch_sample<8, BF16>(p, row, s);
  return launch_sample<32, BF16>(p, 8192, s);
}

}  // namespace grace

extern "C" grace_status_t grace_sample(const float* logits_f32, const uint16_t* logits_bf16, int64_t ld, const uint64_t* allow_bits,
                                       const float* row_score, const float* row_lse, const float* temperature,
                                       const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                                       int B, int M, int V, int draws, float* out_score, float* out_logq,
                                       int32_t* out_parent, int32_t* out_token, int32_t* d_status, void* stream) {
  using namespace grace;
  if ((logits_f32 == nullptr) == (logits_bf16 == nullptr) || !u || !out_score || !out_token) return GRACE_INVALID_ARG;
  if (B <= 0 || M <= 0 || V <= 0 || draws <= 0 || ld < V) return GRACE_INVALID_ARG;
  const uintptr_t words = reinterpret_cast<uintptr_t>(logits_f32) | reinterpret_cast<uintptr_t>(row_score) | reinterpret_cast<uintptr_t>(row_lse) |
                          reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) | reinterpret_cast<uintptr_t>(top_p) |
                          reinterpret_cast<uintptr_t>(min_p) | reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(out_score) |
                          reinterpret_cast<uintptr_t>(out_logq) | reinterpret_cast<uintptr_t>(out_parent) | reinterpret_cast<uintptr_t>(out_token);
  if ((words & 3) || (reinterpret_cast<uintptr_t>(logits_bf16) & 1) || (reinterpret_cast<uintptr_t>(allow_bits) & 7)) return GRACE_INVALID_ARG;
  if (V > kSampleMostV || (int64_t)B * M > 0x7fffffffll) return GRACE_UNSUPPORTED_SHAPE;
  SampleParams p = {};
  const bool bf16 = logits_bf16 != nullptr;
  p.logits = bf16 ? (const void*)logits_bf16 : (const void*)logits_f32;
  p.allow = allow_bits; p.row_score = row_score; p.row_lse = row_lse; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
  p.u = u; p.out_score = out_score; p.out_logq = out_logq; p.out_parent = out_parent; p.out_token = out_token; p.d_status = d_status;
  p.ld = ld; p.R = (int64_t)B * M; p.M = M; p.V = V; p.draws = draws;
  p.vec = ((reinterpret_cast<uintptr_t>(p.logits) | (uintptr_t)(ld * (bf16 ? 2 : 4))) & (bf16 ? 7 : 15)) == 0;
  cudaStream_t s = (cudaStream_t)stream;
  return bf16 ? run_sample<true>(p, s) : run_sample<false>(p, s);
}
