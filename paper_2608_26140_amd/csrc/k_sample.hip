// Sampled commit: one token of each row of logits, drawn by a given number.
//
// The tokens of a row are ordered by logit, equal ones by index; a token's
// weight is exp((x - max) / T), the cuts (top-k, top-p, min-p) each keep a
// prefix of that order, and the token drawn is the first whose cumulative
// weight exceeds u times the kept weight.  So all that is asked of a row are a
// few quantiles of its order, by count or by weight, and no row is sorted: a
// histogram over the logits' bits is refined until one value is left, whose
// tokens have equal weights and are told apart by index.
//
// Weights are held as 64-bit integers, 2^44 for the largest (a row has at most
// 2^19 tokens), computed in fp64: sums of integers do not depend on their order, so
// atomics change nothing, and a draw differs from one in exact arithmetic only
// where u falls within about 2^-44 of the row's weight of a border.
#include "device.h"
#include "internal.h"

namespace acache {

namespace {

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr double kUnit = 17592186044416.0;  // 2^44

struct Settings {
  double inv_t, u, top_p, min_p;
  int top_k;  // n or more: no cut
};

__device__ __forceinline__ Settings settings_of(const SampleRows& r, int64_t row) {
  Settings s;
  const float t = r.temperature ? r.temperature[row] : 1.f;
  const int k = r.top_k ? r.top_k[row] : 0;
  s.top_k = k <= 0 ? r.n : min(k, r.n);
  s.inv_t = 1.0 / (double)fminf(t, 3.4028234663852886e38f);  // an infinite T: all but equal weights
  if (!(t > 0.f)) {  // greedy: the first of the order
    s.inv_t = 1.0;
    s.top_k = 1;
  }
  s.top_p = r.top_p ? (double)r.top_p[row] : 1.0;
  const float mp = r.min_p ? r.min_p[row] : 0.f;
  s.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;
  const double u = r.u[row];
  s.u = u > 0.0 ? fmin(u, 1.0) : 0.0;
  return s;
}

// A logit's weight; m is the row's largest.
__device__ __forceinline__ double weight_of(float x, float m, double inv_t) {
  return x == m ? 1.0 : exp(((double)x - (double)m) * inv_t);
}
__device__ __forceinline__ u64 units_of(double w) { return (u64)rint(w * kUnit); }

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <typename N>
__device__ __forceinline__ N wave_scan(N v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const N t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}

// Element i of a row, fp32 order key (larger key, larger logit; 0: NaN).
template <typename T>
__device__ __forceinline__ float logit_at(const T* x, int i) { return to_f32(x[i]); }

constexpr int kBits = 11, kBins = 1 << kBits;
struct Shared {
  u64 mass[kBins];
  uint32_t count[kBins];
  u64 part_m[kWaves];
  uint32_t part_c[kWaves];
  double part_d[kWaves];
  float part_f[kWaves];
  // what a search found: the bin, what lies before it
  int bin;
  uint32_t before_c, in_c;
  u64 before_m, in_m;
  int seg[1024];
  int found;
};

// A border in the order: the value's key, tokens and weight before it, tokens
// of that value and the weight of each.
struct Border {
  uint32_t key, before_c, in_c;
  u64 before_m, in_m;
};

// Histogram of the row's tokens whose key agrees with `key` above bit
// shift + kBits, by the kBits bits from `shift` on.
template <typename T>
__device__ void histogram(Shared& s, const T* x, int n, float m, double inv_t, uint32_t key, int shift, int bits) {
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    s.mass[i] = 0;
    s.count[i] = 0;
  }
  __syncthreads();
  const int above = shift + bits;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const float v = logit_at(x, i);
    const uint32_t k = order_key(__float_as_uint(v));
    if (k <= 0x007FFFFFu || (above < 32 && (k >> above) != (key >> above))) continue;  // NaN and -inf weigh nothing
    const int bin = (k >> shift) & ((1 << bits) - 1);
    atomicAdd(&s.count[bin], 1u);
    const u64 w = units_of(weight_of(v, m, inv_t));
    if (w) atomicAdd(&s.mass[bin], w);
  }
  __syncthreads();
}

// The bin that holds the border, from the highest down: by count, the one with
// before < want <= before + its count; by weight, likewise with weights.  Past
// the last, the last bin with a token (of weight).
__device__ void search(Shared& s, bool by_mass, uint32_t want_c, u64 want_m, uint32_t base_c, u64 base_m) {
  // thread t takes bins kBins - 1 - 2t and kBins - 2 - 2t
  const int hi = kBins - 1 - 2 * threadIdx.x, lo = hi - 1;
  const uint32_t c0 = s.count[hi], c1 = s.count[lo];
  const u64 m0 = s.mass[hi], m1 = s.mass[lo];
  const int wave = threadIdx.x >> 6;
  const uint32_t ci = wave_scan(c0 + c1);
  const u64 mi = wave_scan(m0 + m1);
  if ((threadIdx.x & 63) == 63) {
    s.part_c[wave] = ci;
    s.part_m[wave] = mi;
  }
  __syncthreads();
  uint32_t bc = base_c + ci - c0 - c1;
  u64 bm = base_m + mi - m0 - m1;
  for (int w = 0; w < wave; ++w) {
    bc += s.part_c[w];
    bm += s.part_m[w];
  }
  auto take = [&](int bin, uint32_t cnt, u64 mass) {
    const bool here = by_mass ? mass > 0 && bm < want_m : cnt > 0 && bc < want_c;
    const bool ends = by_mass ? want_m <= bm + mass : want_c <= bc + cnt;
    if (here && ends) {
      s.bin = bin;
      s.before_c = bc;
      s.before_m = bm;
      s.in_c = cnt;
      s.in_m = mass;
    }
    bc += cnt;
    bm += mass;
  };
  take(hi, c0, m0);
  take(lo, c1, m1);
  __syncthreads();
}

template <typename T>
__device__ Border find(Shared& s, const T* x, int n, float m, double inv_t, bool by_mass, uint32_t want_c, u64 want_m) {
  Border b = {0u, 0u, 0u, 0, 0};
  const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
  for (int level = 0; level < 3; ++level) {
    histogram(s, x, n, m, inv_t, b.key, shifts[level], bits[level]);
    search(s, by_mass, want_c, want_m, b.before_c, b.before_m);
    b.key |= (uint32_t)s.bin << shifts[level];
    b.before_c = s.before_c;
    b.before_m = s.before_m;
    b.in_c = s.in_c;
    b.in_m = s.in_m;
    __syncthreads();
  }
  return b;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_commit_kernel(SampleRows r) {
  __shared__ Shared s;
  const int64_t row = blockIdx.x;
  const T* x = (const T*)r.x + row * r.ld;
  const int n = r.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Settings set = settings_of(r, row);

  // the largest logit
  float m = -INFINITY;
  for (int i = threadIdx.x; i < n; i += kThreads) m = fmaxf(m, logit_at(x, i));
  m = wave_max(m);
  if (lane == 0) s.part_f[wave] = m;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s.part_f[w]);
  int pick = 0;
  float conf = 0.f, prob = 0.f;
  if (m > -INFINITY) {
    // weights of all, of those of at least min_p, and at T = 1
    u64 all = 0, high = 0;
    uint32_t some = 0;
    double soft = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const float v = logit_at(x, i);
      if (!(v > -INFINITY)) continue;
      const double w = weight_of(v, m, set.inv_t);
      const u64 units = units_of(w);
      all += units;
      ++some;
      if (w >= set.min_p) high += units;
      if (r.conf) soft += weight_of(v, m, 1.0);
    }
    auto total = [&](u64 v) {
      v = wave_sum_u64(v);
      __syncthreads();
      if (lane == 0) s.part_m[wave] = v;
      __syncthreads();
      u64 t = 0;
      for (int w = 0; w < kWaves; ++w) t += s.part_m[w];
      return t;
    };
    all = total(all);
    high = total(high);
    const uint32_t valid = (uint32_t)total(some);
    soft = wave_sum_f64(soft);
    if (lane == 0) s.part_d[wave] = soft;
    __syncthreads();
    soft = 0.0;
    for (int w = 0; w < kWaves; ++w) soft += s.part_d[w];

    u64 kept = all;
    if (set.top_k < (int)valid) {
      const Border b = find(s, x, n, m, set.inv_t, false, (uint32_t)set.top_k, 0);
      kept = b.before_m + (u64)(set.top_k - b.before_c) * (b.in_m / b.in_c);
    }
    if (set.top_p < 1.0) {
      const double want = fmax(set.top_p, 0.0) * (double)kept;
      const u64 least = min(max((u64)1, (u64)ceil(want)), kept);
      const Border b = find(s, x, n, m, set.inv_t, true, 0, least);
      const u64 each = b.in_m / b.in_c;
      kept = min(kept, b.before_m + (least - b.before_m + each - 1) / each * each);
    }
    kept = min(kept, max(high, units_of(1.0)));
    const u64 target = min((u64)(set.u * (double)kept), kept - 1);
    const Border b = find(s, x, n, m, set.inv_t, true, 0, target + 1);
    const u64 each = b.in_m / b.in_c;
    int nth = (int)((target - b.before_m) / each);
    const float value = __uint_as_float((b.key & 0x80000000u) ? b.key & 0x7FFFFFFFu : ~b.key);
    prob = (float)((double)each / (double)kept);
    conf = (float)(weight_of(value, m, 1.0) / soft);
    // the nth token of that value
    const int seg = (n + 1023) / 1024;  // of 1024 tokens
    for (int i = threadIdx.x; i < seg; i += kThreads) s.seg[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint64_t same = __ballot(order_key(__float_as_uint(logit_at(x, i))) == b.key);
      if (same && lane == __ffsll((unsigned long long)__ballot(1)) - 1) atomicAdd(&s.seg[i >> 10], __popcll(same));
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int at = 0;
      while (at + 1 < seg && nth >= s.seg[at]) nth -= s.seg[at++];
      for (int i = at * 1024; i < min(n, at * 1024 + 1024); ++i)
        if (order_key(__float_as_uint(logit_at(x, i))) == b.key && nth-- == 0) {
          s.found = i;
          break;
        }
    }
    __syncthreads();
    pick = s.found;
  } else {
    // nothing to draw from: the lowest index among the largest, NaN lowest
    int best = n;
    for (int i = threadIdx.x; i < n; i += kThreads)
      if (logit_at(x, i) == -INFINITY) best = min(best, i);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = min(best, __shfl_xor(best, o));
    __syncthreads();
    if (lane == 0) s.seg[wave] = best;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) best = min(best, s.seg[w]);
    pick = best < n ? best : 0;
  }
  if (threadIdx.x == 0) {
    r.out[row] = pick;
    if (r.conf) r.conf[row] = conf;
    if (r.prob) r.prob[row] = prob;
    if (r.commit_pos) {
      const int64_t at = r.commit_pos[row];
      if (at >= 0 && at < r.ids_len) r.ids[at] = pick;
    }
  }
}

}  // namespace

hipError_t launch_sample_commit(acache_dtype dt, const SampleRows& r, int rows, hipStream_t s) {
  if (dt == ACACHE_BF16) hipLaunchKernelGGL(sample_commit_kernel<bf16>, dim3(rows), dim3(kThreads), 0, s, r);
  else hipLaunchKernelGGL(sample_commit_kernel<float>, dim3(rows), dim3(kThreads), 0, s, r);
  return hipGetLastError();
}

}  // namespace acache
