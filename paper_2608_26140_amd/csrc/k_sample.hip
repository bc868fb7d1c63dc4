// Sampled commit: one token of each row of logits, drawn by a given number.
//
// The tokens of a row are ordered by logit, equal ones by index; a token's
// weight is exp((x - max) / T), the cuts (top-k, top-p, min-p) each keep a
// prefix of that order, and the token drawn is the first whose cumulative
// weight exceeds u times the kept weight.  So all that is asked of a row are a
// few borders of its order, by count or by weight, and no row is sorted.
//
// Weights are held as 64-bit integers, 2^44 for the largest (a row has at most
// 2^19 tokens), computed in fp64: sums of integers do not depend on their order, so
// atomics change nothing, and a draw differs from one in exact arithmetic only
// where u falls within about n 2^-44 of the row's weight of a border.
//
// The kernels take a row as a histogram over the upper 16 bits of its logits,
// one bin for each such value of magnitude 2^-27 to 512 and one for what lies
// between, mostly zeros, in LDS.  Of bf16 logits a bin's tokens are equal: its
// weight is its count times one exponential, and a border in the bin is a
// division.  Of fp32 logits a bin sums its tokens' weights, and a border is then
// looked for among its tokens.  Rows with logits of 512 and more, with a border
// among the smallest ones when they are not all zeros, bf16 rows with more than
// kSmall nonzero ones of these, and fp32 rows with more than 1024 tokens of
// several values in a border's bin go by sample_any, which refines a histogram
// over the logits' order keys and reads the row anew for each step.  A call of 1024
// bf16 rows of 126464 takes 720 to 870 us with one such row, 79 without, one of 67
// fp32 rows of 50021 108 and 44.  Of normally distributed logits some 10^-9 are
// nonzero and below 2^-27, which is why these have a place of their own; fp32 logits
// far from zero crowd a bin (67 rows of 126464 of spread 2.5: 93 us around 0, 100
// around 5, 380 around 10, 430 around 20).
#include "device.h"
#include "internal.h"

namespace acache {

namespace {

typedef unsigned long long u64;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;
typedef __attribute__((__vector_size__(2 * sizeof(int16_t)))) int16_t i16x2;
constexpr int kMaxThreads = 1024, kMaxWaves = kMaxThreads / 64;
constexpr double kScaleOne = 64 * 1.4426950408889634;  // 64 log2(e)

struct Settings {
  double scale;  // 64 log2(e) / T
  double u, top_p, min_p;
  int top_k;     // n or more: no cut
};

__device__ __forceinline__ Settings settings_of(const SampleRows& r, int64_t row) {
  Settings s;
  const float t = r.temperature ? r.temperature[row] : 1.f;
  const int k = r.top_k ? r.top_k[row] : 0;
  s.top_k = k <= 0 ? r.n : min(k, r.n);
  s.scale = kScaleOne / (double)fminf(t, 3.4028234663852886e38f);  // an infinite T: all but equal weights
  if (!(t > 0.f)) {  // greedy: the first of the order
    s.scale = kScaleOne;
    s.top_k = 1;
  }
  s.top_p = r.top_p ? (double)r.top_p[row] : 1.0;
  const float mp = r.min_p ? r.min_p[row] : 0.f;
  s.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;
  const double u = r.u[row];
  s.u = u > 0.0 ? fmin(u, 1.0) : 0.0;
  return s;
}

// exp(d scale) for d <= 0 in fp64, scale given in 64ths of a power of two: the
// nearest 64th from a table, the rest by the exponential series to degree 4 (its
// next term, 0.0054^5 / 120, is 4e-14 of the result).  At least 2^-1000.
struct Table {
  double at[64];
};
__device__ __forceinline__ void fill(Table& t) {
  if (threadIdx.x < 64) t.at[threadIdx.x] = exp2((double)threadIdx.x / 64.0);
}
__device__ __forceinline__ double exp_down(const Table& t, double d, double scale) {
  constexpr double kNearest = 6755399441055744.0;  // 1.5 2^52: adding it rounds to a whole number
  constexpr double c1 = 0.6931471805599453 / 64, c2 = c1 * c1 / 2, c3 = c2 * c1 / 3, c4 = c3 * c1 / 4;
  const double y = fmax(d * scale, -64000.0), z = y + kNearest;
  const int k = (int)(uint32_t)__double_as_longlong(z);
  const double f = y - (z - kNearest);
  const double p = fma(fma(fma(fma(c4, f, c3), f, c2), f, c1), f, 1.0) * t.at[k & 63];
  return __longlong_as_double(__double_as_longlong(p) + ((long long)((k & ~63) << 14) << 32));
}
// w 2^44 rounded, for w <= 1: 256 + w has steps of 2^-44.
__device__ __forceinline__ u64 units_of(double w) { return (u64)__double_as_longlong(w + 256.0) - 0x4070000000000000ull; }

// Sums across a wave by moves within its registers (DPP): shifts by 1, 2, 4 and
// 8 in rows of 16 lanes, then the rows' last lanes to the rows behind.  A shuffle
// through LDS takes several times as long, and these stand one behind the other.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 v) {
  return (u64)moved<CTRL, ROWS>((uint32_t)v) | (u64)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {
  return __longlong_as_double((long long)moved<CTRL, ROWS>((u64)__double_as_longlong(v)));
}
template <typename N>
__device__ __forceinline__ N wave_scan(N v) {  // inclusive
  v += moved<0x111, 0xF>(v);
  v += moved<0x112, 0xF>(v);
  v += moved<0x114, 0xF>(v);
  v += moved<0x118, 0xF>(v);
  v += moved<0x142, 0xA>(v);  // lane 15 of rows 0 and 2 to rows 1 and 3
  v += moved<0x143, 0xC>(v);  // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
  return (u64)lane_of((uint32_t)v, lane) | (u64)lane_of((uint32_t)(v >> 32), lane) << 32;
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  return __longlong_as_double((long long)lane_of((u64)__double_as_longlong(v), lane));
}
template <typename N>
__device__ __forceinline__ N wave_total(N v) {
  return lane_of(wave_scan(v), 63);
}

__device__ __forceinline__ void write_pick(const SampleRows& r, int64_t row, int pick, double conf, double prob) {
  r.out[row] = pick;
  if (r.conf) r.conf[row] = (float)conf;
  if (r.prob) r.prob[row] = (float)prob;
  if (r.commit_pos) {
    const int64_t at = r.commit_pos[row];
    if (at >= 0 && at < r.ids_len) r.ids[at] = pick;
  }
}

__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
  v = max(v, moved<0x111, 0xF>(v));
  v = max(v, moved<0x112, 0xF>(v));
  v = max(v, moved<0x114, 0xF>(v));
  v = max(v, moved<0x118, 0xF>(v));
  v = max(v, moved<0x142, 0xA>(v));
  v = max(v, moved<0x143, 0xC>(v));
  return lane_of(v, 63);
}

// An entry of an ordered list of (count, weight) and what lies before it.
struct Border {
  int at;
  uint32_t before_c, in_c;
  u64 before_m, in_m;
};

// n / each rounded down, n < each 2^19: the quotient in fp64 is off by one at most.
__device__ __forceinline__ uint32_t whole_times(u64 n, u64 each) {
  uint32_t q = (uint32_t)((double)n / (double)each);
  if (q * each > n) --q;
  if ((q + 1) * each <= n) ++q;
  return q;
}

// The entry with before < want <= before + its own, by count or by weight, run
// by one wave on N entries a lane; the bases count as before the first.  By
// weight, what is counted before it is left out.
template <int N, typename C, typename M>
__device__ __forceinline__ Border find_entry(bool by_mass, uint32_t want_c, u64 want_m, uint32_t base_c, u64 base_m,
                                             C count_at, M mass_at) {
  const int lane = threadIdx.x & 63;
  uint32_t c[N], cs = 0;
  u64 m[N], ms = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = count_at(lane * N + i);
    m[i] = mass_at(lane * N + i);
    cs += c[i];
    ms += m[i];
  }
  u64 bm = base_m + wave_scan(ms) - ms;
  uint32_t bc = 0;
  u64 who;
  if (by_mass) {
    who = __ballot(bm < want_m && want_m <= bm + ms);
  } else {
    bc = base_c + wave_scan(cs) - cs;
    who = __ballot(bc < want_c && want_c <= bc + cs);
  }
  if (!who) return {0, 0, 0, 0, 0};
  const int src = __ffsll(who) - 1;
  Border f = {src * N, lane_of(bc, src), lane_of(c[0], src), lane_of(bm, src), lane_of(m[0], src)};
#pragma unroll
  for (int i = 1; i < N; ++i) {
    const bool past = by_mass ? want_m > f.before_m + f.in_m : want_c > f.before_c + f.in_c;
    if (past) f = {src * N + i, f.before_c + f.in_c, lane_of(c[i], src), f.before_m + f.in_m, lane_of(m[i], src)};
  }
  return f;
}

// m / c where that is whole (equal tokens), at most 2^45: the quotient in fp64,
// of a product that may have more than 53 bits, is less than 1/2 off.
__device__ __forceinline__ u64 whole_of(u64 m, uint32_t c) { return (u64)rint((double)m / (double)c); }

// The three borders of a row in their turn; the search is given.  kept: the
// weight of all tokens; high: of those of at least min_p.  The last border is
// the drawn value's, nth the token among those of that value.
struct Draw {
  Border at;
  uint32_t nth;
  double prob;
};
template <typename F>
__device__ __forceinline__ Draw draw_by(const Settings& set, u64 kept, u64 high, uint32_t valid, F border) {
  Draw d = {{0, 0, 1, 0, 1}, 0, 0.0};
#pragma unroll 1
  for (int cut = 0; cut < 3; ++cut) {  // top-k, top-p, the draw
    if (cut == 0 && set.top_k >= (int)valid) continue;
    if (cut == 1 && !(set.top_p < 1.0)) continue;
    u64 want = 0;
    if (cut == 1) want = min(max((u64)1, (u64)ceil(fmax(set.top_p, 0.0) * (double)kept)), kept);
    if (cut == 2) {
      kept = min(kept, max(high, units_of(1.0)));
      want = min((u64)(set.u * (double)kept), kept - 1) + 1;
    }
    d.at = border(cut, (uint32_t)set.top_k, want);
    if (d.at.in_c == 0) return d;
    const u64 each = d.at.in_c == 1 ? d.at.in_m : whole_of(d.at.in_m, d.at.in_c);
    if (cut == 0) kept = d.at.before_m + (u64)(set.top_k - d.at.before_c) * each;
    if (cut == 1) kept = min(kept, d.at.before_m + (whole_times(want - d.at.before_m - 1, each) + 1) * each);
    if (cut == 2) {
      d.nth = whole_times(want - 1 - d.at.before_m, each);
      d.prob = (double)each / (double)kept;
    }
  }
  return d;
}

// ---------------------------------------------------------------- any row
constexpr int kAnyBins = 2048;
struct Any {
  Table table;
  u64 mass[kAnyBins];
  uint32_t count[kAnyBins];
  u64 part_m[kMaxWaves];
  double part_d[kMaxWaves];
  float part_f[kMaxWaves];
  Border found;
  int seg[512];
  int at;
};

template <typename T>
__device__ void sample_any(Any& s, const SampleRows& r, int64_t row) {
  const T* x = (const T*)r.x + row * r.ld;
  const int n = r.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const Settings set = settings_of(r, row);
  // infinities: a largest of +inf weighs 1, and all below it nothing
  auto weight_of = [&](float v, float m, double scale) { return v == m ? 1.0 : exp_down(s.table, (double)v - (double)m, scale); };
  auto key_at = [&](int i) { return order_key(__float_as_uint(to_f32(x[i]))); };
  constexpr uint32_t kNothing = 0x007FFFFFu;  // -inf's key; NaN's is 0

  float m = -INFINITY;
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += (int)blockDim.x) m = fmaxf(m, to_f32(x[i]));
  m = wave_max(m);
  __syncthreads();
  fill(s.table);
  if (lane == 0) s.part_f[wave] = m;
  __syncthreads();
  for (int w = 0; w < waves; ++w) m = fmaxf(m, s.part_f[w]);
  if (m == -INFINITY) {  // nothing to draw from: the lowest index among the largest, NaN lowest
    if (threadIdx.x == 0) s.at = n;
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += (int)blockDim.x)
      if (to_f32(x[i]) == -INFINITY) atomicMin(&s.at, i);
    __syncthreads();
    if (threadIdx.x == 0) write_pick(r, row, s.at < n ? s.at : 0, 0.0, 0.0);
    return;
  }
  u64 all = 0, high = 0, some = 0;
  double soft = 0.0;
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += (int)blockDim.x) {
    const float v = to_f32(x[i]);
    if (!(v > -INFINITY)) continue;
    const double w = weight_of(v, m, set.scale);
    all += units_of(w);
    if (w >= set.min_p) high += units_of(w);
    ++some;
    if (r.conf) soft += weight_of(v, m, kScaleOne);
  }
  auto total = [&](u64 v) {
    v = wave_total(v);
    __syncthreads();
    if (lane == 0) s.part_m[wave] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < waves; ++w) v += s.part_m[w];
    return v;
  };
  all = total(all);
  high = total(high);
  some = total(some);
  soft = wave_total(soft);
  if (lane == 0) s.part_d[wave] = soft;
  __syncthreads();
  soft = 0.0;
  for (int w = 0; w < waves; ++w) soft += s.part_d[w];

  uint32_t key = 0;
  const Draw d = draw_by(set, all, high, (uint32_t)some, [&](int cut, uint32_t want_c, u64 want_m) {
    // the key's bits from the top: 11, 11 and 10 at a time
    Border b = {0, 0, 0, 0, 0};
    key = 0;
#pragma unroll 1
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift == 10 ? 0 : -1) {
      const int bits = shift ? 11 : 10;
#pragma unroll 1
      for (int i = threadIdx.x; i < kAnyBins; i += (int)blockDim.x) {
        s.mass[i] = 0;
        s.count[i] = 0;
      }
      __syncthreads();
#pragma unroll 1
      for (int i = threadIdx.x; i < n; i += (int)blockDim.x) {
        const uint32_t k = key_at(i);
        if (k <= kNothing || (shift < 21 && (k >> (shift + bits)) != (key >> (shift + bits)))) continue;
        const int bin = kAnyBins - 1 - ((k >> shift) & ((1 << bits) - 1));  // largest first
        atomicAdd(&s.count[bin], 1u);
        const u64 w = units_of(weight_of(to_f32(x[i]), m, set.scale));
        if (w) atomicAdd(&s.mass[bin], w);
      }
      __syncthreads();
      if (wave == 0) {
        // 32 runs of 64 bins: the run, then the bin
        u64 run_m = 0;
        uint32_t run_c = 0;
#pragma unroll 1
        for (int g = 0; g < 32; ++g) {
          const u64 mt = wave_total(s.mass[g * 64 + lane]);
          const uint32_t ct = wave_total(s.count[g * 64 + lane]);
          if (lane == g) {
            run_m = mt;
            run_c = ct;
          }
        }
        Border f = find_entry<1>(cut != 0, want_c, want_m, b.before_c, b.before_m, [&](int) { return run_c; },
                                 [&](int) { return run_m; });
        const int g = f.at * 64;
        f = find_entry<1>(cut != 0, want_c, want_m, f.before_c, f.before_m, [&](int i) { return s.count[g + i]; },
                          [&](int i) { return s.mass[g + i]; });
        f.at += g;
        if (lane == 0) s.found = f;
      }
      __syncthreads();
      b = s.found;
      key |= (uint32_t)(kAnyBins - 1 - b.at) << shift;
      __syncthreads();
    }
    return b;
  });
  // the nth token of that value, by segments of 1024 tokens
  uint32_t nth = d.nth;
  const int seg = (n + 1023) / 1024;
  for (int i = threadIdx.x; i < seg; i += (int)blockDim.x) s.seg[i] = 0;
  __syncthreads();
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += (int)blockDim.x)
    if (key_at(i) == key) atomicAdd(&s.seg[i >> 10], 1);
  __syncthreads();
  int at = 0;
  while (at + 1 < seg && nth >= (uint32_t)s.seg[at]) nth -= s.seg[at++];
  if (wave == 0) {
#pragma unroll 1
    for (int i0 = at * 1024; i0 < min(n, at * 1024 + 1024); i0 += 64) {
      const bool same = i0 + lane < n && key_at(i0 + lane) == key;
      const uint32_t here = __popcll(__ballot(same)), before = __popcll(__ballot(same) & ((1ull << lane) - 1));
      if (same && before == nth)
        write_pick(r, row, i0 + lane, weight_of(to_f32(x[i0 + lane]), m, kScaleOne) / soft, d.prob);
      if (nth < here) break;
      nth -= here;
    }
  }
}

// ---------------------------------------------------------------- by bins
constexpr int kLow = 100 << 7, kRange = (136 - 100) << 7;  // upper halves of 2^-27 .. 512
constexpr int kValues = 2 * kRange + 1;
constexpr int kGroups = (kValues + 127) / 128;             // of 128 bins, two a lane
constexpr int kBins = kGroups * 128;
static_assert(kGroups <= 128, "two groups a lane");

// Bins are numbered in the order of the values, largest first, zeros and what is
// below 2^-27 are bin kRange; in memory the positive ones lie in ascending order.
__device__ __forceinline__ int place_of(int bin) { return bin < kRange ? kRange - 1 - bin : bin; }
__device__ __forceinline__ uint32_t half_of_bin(int bin) {
  const uint32_t off = bin < kRange ? kRange - 1 - bin : bin - kRange - 1;
  return bin == kRange ? 0u : (off + kLow) | (bin < kRange ? 0u : 0x8000u);
}
__device__ __forceinline__ float value_of_bin(int bin) { return __uint_as_float(half_of_bin(bin) << 16); }

// What lies outside the bins: NaN and -inf weigh nothing (0); a negative of 512
// and more weighs nothing beside a largest logit well above (2, see by_bins); a
// positive one is for sample_any (1).
constexpr uint32_t kElsewhere = 1, kFarBelow = 2;
__device__ __forceinline__ uint32_t outside(uint32_t bits) {
  if ((bits & 0x7FFFFFFFu) > 0x7F800000u || bits == 0xFF800000u) return 0;
  return !(bits & 0x80000000u) ? kElsewhere : kFarBelow;
}
// What is left out may weigh e^-60 of the largest at most, so that a whole row of
// 2^19 such tokens is 2^23 times less than a unit: at the temperature drawn with
// and, where the confidence is asked for, at 1, whichever makes more of them.
__device__ __forceinline__ bool by_bins(uint32_t flags, float m, double scale, bool conf) {
  if (conf) scale = fmin(scale, kScaleOne);
  return !(flags & kElsewhere) && m > -512.f && (!(flags & kFarBelow) || ((double)m + 512.0) * scale > 60.0 * kScaleOne);
}

// A row in 16-byte pieces at their own alignment; what a piece holds outside
// the row counts as NaN.
template <typename T>
struct Pieces {
  static constexpr int PER = 16 / sizeof(T);
  const T* x;
  int n, skew, rounds;
  __device__ __forceinline__ Pieces(const T* row, int len) : x(row), n(len) {
    skew = (int)(((uintptr_t)row & 15) / sizeof(T));
    rounds = (n + skew + PER * (int)blockDim.x - 1) / (PER * (int)blockDim.x);
  }
  __device__ __forceinline__ int index(int round, int j) const { return (round * (int)blockDim.x + (int)threadIdx.x) * PER + j - skew; }
  __device__ __forceinline__ u32x4 fetch(int round) const {
    const int at = index(round, 0);
    if (at >= 0 && at + PER <= n) return *reinterpret_cast<const u32x4*>(x + at);
    u32x4 v = {~0u, ~0u, ~0u, ~0u};
    if (at > -PER && at < n) {
      T t[PER];
      __builtin_memcpy(t, &v, 16);
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (at + j >= 0 && at + j < n) t[j] = x[at + j];
      __builtin_memcpy(&v, t, 16);
    }
    return v;
  }
  // f(round, piece) for every round in turn, uniform over the workgroup, four
  // pieces on their way at a time, the first ones asked for by begin(); rounds
  // that lie within the row need no look at its ends
  struct Ahead {
    u32x4 v[4];
  };
  __device__ __forceinline__ const u32x4* whole() const { return reinterpret_cast<const u32x4*>(x - skew) + threadIdx.x; }
  __device__ __forceinline__ int first_whole() const { return skew ? 1 : 0; }
  __device__ __forceinline__ int end_whole() const { return (n + skew) / (PER * (int)blockDim.x); }
  __device__ __forceinline__ Ahead begin() const {
    Ahead a;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      a.v[i] = first_whole() + 4 <= end_whole() ? whole()[(first_whole() + i) * (int)blockDim.x] : u32x4{0, 0, 0, 0};
    return a;
  }
  template <typename F>
  __device__ __forceinline__ void each(Ahead a, F f) const {
    const int end = end_whole();
    int c = first_whole();
    if (c) f(0, fetch(0));
    if (c + 4 <= end) {
#pragma unroll 1
      for (; c + 8 <= end; c += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // a piece is taken and the one four rounds on asked for
          const u32x4 now = a.v[i];
          a.v[i] = whole()[(c + 4 + i) * (int)blockDim.x];
          f(c + i, now);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) f(c + i, a.v[i]);
      c += 4;
    }
#pragma unroll 1
    for (; c < rounds; ++c) f(c, fetch(c));
  }
  // the same for longer f: one copy of it, the next piece on its way
  template <typename F>
  __device__ __forceinline__ void each_long(F f) const {
    u32x4 v = fetch(0);
#pragma unroll 1
    for (int c = 0; c < rounds; ++c) {
      const u32x4 now = v;
      if (c + 1 < rounds) v = fetch(c + 1);
      f(c, now);
    }
  }
};

struct Bins {
  Table table;
  uint32_t count[kBins];
  uint32_t group_c[128];
  u64 group_m[128];
  u64 part_m[kMaxWaves];
  double part_d[kMaxWaves];
  float part_f[kMaxWaves];
  uint32_t flags;
  int first;
};

__device__ __forceinline__ void clear(Bins& s) {
  fill(s.table);
  for (int i = threadIdx.x; i < kBins; i += (int)blockDim.x) s.count[i] = 0;
  for (int i = threadIdx.x; i < 128; i += (int)blockDim.x) {
    s.group_c[i] = 0;
    s.group_m[i] = 0;
  }
  if (threadIdx.x == 0) {
    s.flags = 0;
    s.first = kBins;
  }
}

// The bin of a border; mass_at gives a bin's weight.
template <typename M>
__device__ __forceinline__ Border find_bin(const Bins& s, bool by_mass, uint32_t want_c, u64 want_m, M mass_at) {
  Border f = find_entry<2>(by_mass, want_c, want_m, 0, 0, [&](int i) { return s.group_c[i]; },
                           [&](int i) { return s.group_m[i]; });
  const int g = f.at * 128;
  f = find_entry<2>(by_mass, want_c, want_m, f.before_c, f.before_m, [&](int i) { return s.count[place_of(g + i)]; },
                    [&](int i) { return mass_at(g + i); });
  f.at += g;
  return f;
}

// Adds up what every thread has.
__device__ __forceinline__ void gather_sums(Bins& s, u64& high, double& soft) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  high = wave_total(high);
  soft = wave_total(soft);
  if (lane == 0) {
    s.part_m[wave] = high;
    s.part_d[wave] = soft;
  }
  __syncthreads();
  high = wave_total(lane < waves ? s.part_m[lane] : (u64)0);
  soft = wave_total(lane < waves ? s.part_d[lane] : 0.0);
}

// bf16: one read of the row into the histogram, exponentials of the bins that
// have tokens, the borders by one wave, and a second read for the token's index.
// Bound by its vector instructions, 14 a logit: with 1024 rows (78 us) they take 75%
// of the SIMDs' cycles at four each, and the LDS works in 44% of a CU's (28% are
// bank conflicts of the atomics, one a logit); a row of 126464, 21.8 us, on one CU:
// 51% and 30%.  What is outside the bins, masked logits among it, adds to one place:
// 1024 rows with 90% of -inf or of the type's lowest value take 410 us.
constexpr int kSmall = 16;
struct BinsBf16 {
  Bins b;
  uint32_t zeros, half, nth, top;
  uint32_t small_n, mixed;  // nonzero logits below the bins; set if a border lies among them
  uint16_t small[kSmall];
  u64 small_m;              // their weight
  double conf, prob;
};
static_assert(sizeof(BinsBf16) <= 40960, "four workgroups a CU");
template <int NT, int WAVES_PER_SIMD>
__global__ __launch_bounds__(NT, WAVES_PER_SIMD) void sample_bf16_kernel(SampleRows r) {
  __shared__ union {
    BinsBf16 f;
    Any any;
  } sh;
  BinsBf16& s = sh.f;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const Pieces<bf16> x((const bf16*)r.x + row * r.ld, r.n);
  const auto ahead = x.begin();
  const Settings set = settings_of(r, row);
  clear(s.b);
  if (threadIdx.x == 0) {
    s.zeros = 0;
    s.top = 0;
    s.small_n = s.mixed = 0;
    s.small_m = 0;
  }
  __syncthreads();

  // Two logits at a time in 16-bit halves: magnitude less kLow, at most kRange,
  // which stands for all that is outside the bins; then the bin, negatives
  // behind the zeros.  Beside it each thread keeps the largest bits, as whole
  // numbers with a sign, of each quarter of its pieces: a value above them is
  // not there, which spares the second read most of the row.
  uint32_t flags = 0;
  const int quarter = (x.rounds + 3) / 4;
  u64 tops = 0;  // of the quarters, the last one lowest
  i16x2 top = {-32768, -32768};
  int left = quarter;
  uint32_t largest = 0;  // of the bits that are positive
  x.each(ahead, [&](int round, const u32x4& v) {
    if (x.index(round, 0) < r.n) {
      u16x2 most = {0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t word = v[j];
        const u16x2 w = __builtin_bit_cast(u16x2, word), sign = w >> (u16x2){15, 15};
        const u16x2 off = __builtin_elementwise_min((w & (u16x2){0x7FFF, 0x7FFF}) - (u16x2){kLow, kLow}, (u16x2){kRange, kRange});
        top = __builtin_elementwise_max(top, __builtin_bit_cast(i16x2, word));
        most = __builtin_elementwise_max(most, off);
        const uint32_t at = __builtin_bit_cast(uint32_t, off + sign * (u16x2){kRange + 1, kRange + 1});
        atomicAdd(&s.b.count[at & 0xFFFFu], 1u);
        atomicAdd(&s.b.count[at >> 16], 1u);
      }
      if (max(most[0], most[1]) == kRange) {  // zeros, and what else is outside
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
          const uint32_t p = ((j < 4 ? j < 2 ? v[0] : v[1] : j < 6 ? v[2] : v[3]) >> (16 * (j & 1))) & 0xFFFFu;
          if ((p & 0x7FFFu) == 0) {
            atomicAdd(&s.zeros, 1u);
          } else if ((p & 0x7FFFu) < (uint32_t)kLow) {
            const uint32_t at = atomicAdd(&s.small_n, 1u);
            if (at < (uint32_t)kSmall) s.small[at] = (uint16_t)p;
            else flags |= kElsewhere;
          } else if ((p & 0x7FFFu) - (uint32_t)kLow >= (uint32_t)kRange) {
            flags |= outside(p << 16);
          }
        }
      }
    }
    if (--left == 0 || round == x.rounds - 1) {
      const int16_t t = max(top[0], top[1]);
      tops = tops << 16 | (uint16_t)t;
      largest = max(largest, (uint32_t)max((int)t, 0));
      top = (i16x2){-32768, -32768};
      left = quarter;
    }
  });
  largest = wave_most(largest);
  if (lane == 0) atomicMax(&s.top, largest);
  if (flags) atomicOr(&s.b.flags, flags);
  __syncthreads();
  if (threadIdx.x == 0) {
    s.b.count[kRange] = s.zeros + s.small_n;
    s.b.count[kValues] = 0;
  }
  float m = __uint_as_float(s.top << 16);
  const bool known = s.top - (uint32_t)kLow < (uint32_t)kRange;  // or no logit, none above 0, or NaN among them
  __syncthreads();
  if (!known) {
#pragma unroll 1
    for (int g = wave; g < kGroups; g += waves) {  // the largest logit's bin
      const uint32_t c0 = s.b.count[place_of(g * 128 + 2 * lane)], c1 = s.b.count[place_of(g * 128 + 2 * lane + 1)];
      const u64 any = __ballot((c0 | c1) != 0);
      if (any) {
        if (lane == __ffsll(any) - 1) atomicMin(&s.b.first, g * 128 + 2 * lane + (c0 == 0));
        break;
      }
    }
    __syncthreads();
    m = s.b.first < kValues ? value_of_bin(s.b.first) : -INFINITY;
  }
  const bool small_top = m == 0.f && s.small_n != 0;
  if (small_top || !by_bins(s.b.flags, m, set.scale, r.conf != nullptr)) {
    __syncthreads();
    sample_any<bf16>(sh.any, r, row);
    return;
  }
  u64 high = 0;
  double soft = 0.0;
  if (s.small_n) {
    if (threadIdx.x < s.small_n) {
      const double d = (double)__uint_as_float((uint32_t)s.small[threadIdx.x] << 16) - (double)m;
      const double w = exp_down(s.b.table, d, set.scale);
      atomicAdd(&s.small_m, units_of(w));
      if (w >= set.min_p) high += units_of(w);
      if (r.conf) soft += exp_down(s.b.table, d, kScaleOne);
    }
    __syncthreads();
  }
#pragma unroll 1
  for (int g = wave; g < kGroups; g += waves) {
    const int bin = g * 128 + 2 * lane;
    const uint32_t c[2] = {s.b.count[place_of(bin)], s.b.count[place_of(bin + 1)]};
    if (!__ballot((c[0] | c[1]) != 0)) continue;
    u64 mass = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (c[i]) {
        const double d = (double)value_of_bin(bin + i) - (double)m;
        const double w = exp_down(s.b.table, d, set.scale);
        const uint32_t n = bin + i == kRange ? s.zeros : c[i];
        const u64 own = n * units_of(w);
        mass += own;
        if (w >= set.min_p) high += own;
        if (r.conf) soft += n * exp_down(s.b.table, d, kScaleOne);
        if (bin + i == kRange) mass += s.small_m;
      }
    const u64 mt = wave_total(mass);
    const uint32_t ct = wave_total(c[0] + c[1]);
    if (lane == 0) {
      s.b.group_c[g] = ct;
      s.b.group_m[g] = mt;
    }
  }
  gather_sums(s.b, high, soft);
  if (wave == 0) {
    u64 all = 0;
    uint32_t valid = 0;
    for (int g = lane; g < 128; g += 64) {
      all += s.b.group_m[g];
      valid += s.b.group_c[g];
    }
    const Draw d = draw_by(set, wave_total(all), high, wave_total(valid),
                           [&](int cut, uint32_t want_c, u64 want_m) -> Border {
                             const Border f = find_bin(s.b, cut != 0, want_c, want_m, [&](int bin) -> u64 {
                               const uint32_t c = bin == kRange ? s.zeros : s.b.count[place_of(bin)];
                               const u64 own = c ? c * units_of(exp_down(s.b.table, (double)value_of_bin(bin) - (double)m, set.scale)) : 0;
                               return bin == kRange ? own + s.small_m : own;
                             });
                             return f.at == kRange && s.small_n != 0 ? Border{0, 0, 0, 0, 0} : f;
                           });
    if (lane == 0) {
      s.mixed = d.at.in_c == 0;
      s.half = half_of_bin(d.at.at);
      s.nth = d.nth;
      s.prob = d.prob;
      s.conf = exp_down(s.b.table, (double)value_of_bin(d.at.at) - (double)m, kScaleOne) / soft;
    }
  }
  __syncthreads();
  if (s.mixed) {
    __syncthreads();
    sample_any<bf16>(sh.any, r, row);
    return;
  }

  // the nth token of that value: counted by round and wave in the counts' place,
  // then within a wave's pieces of one round
  uint32_t* same = s.b.count;
  for (int i = threadIdx.x; i < x.rounds * waves; i += (int)blockDim.x) same[i] = 0;
  __syncthreads();
  const uint32_t half = s.half;
  uint32_t nth = s.nth;
  auto matches = [&](const u32x4& v) {
    uint32_t mask = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t p = (v[j >> 1] >> (16 * (j & 1))) & 0xFFFFu;
      if (p == half || (half == 0 && p == 0x8000u)) mask |= 1u << j;
    }
    return mask;
  };
  const u16x2 half2 = {(uint16_t)half, (uint16_t)half}, bits = half ? (u16x2){0xFFFF, 0xFFFF} : (u16x2){0x7FFF, 0x7FFF};
  const int quarters = (x.rounds + quarter - 1) / quarter;
#pragma unroll 1
  for (int part = 0; part < quarters; ++part) {
    const bool may = half == 0 || (int16_t)(tops >> (16 * (quarters - 1 - part))) >= (int16_t)half;
    if (!__ballot(may)) continue;
    const int end = min(x.rounds, (part + 1) * quarter);
#pragma unroll 1
    for (int c = part * quarter; c < end; c += 4) {
      u32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = may && c + i < end ? x.fetch(c + i) : u32x4{~0u, ~0u, ~0u, ~0u};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u16x2 least = {0xFFFF, 0xFFFF};  // 0 in a half: equal
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t word = v[i][j];
          least = __builtin_elementwise_min(least, (__builtin_bit_cast(u16x2, word) ^ half2) & bits);
        }
        if (__ballot(least[0] == 0 || least[1] == 0)) {
          const uint32_t total = wave_total((uint32_t)__popc(matches(v[i])));
          if (lane == 0) same[(c + i) * waves + wave] = total;
        }
      }
    }
  }
  __syncthreads();
  const int entries = x.rounds * waves;
  int hit = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < entries; i0 += 64) {
    const uint32_t c = i0 + lane < entries ? same[i0 + lane] : 0;
    const uint32_t upto = wave_scan(c);
    const u64 who = __ballot(upto > nth);
    if (who) {
      const int src = __ffsll(who) - 1;
      hit = i0 + src;
      nth -= lane_of(upto - c, src);
      break;
    }
    nth -= lane_of(upto, 63);
  }
  if (wave != hit % waves) return;
  const int round = hit / waves;
  const uint32_t mask = matches(x.fetch(round));
  const uint32_t c = __popc(mask), upto = wave_scan(c);
  if (upto > nth && upto - c <= nth) {
    uint32_t left = mask;
    for (uint32_t k = nth - (upto - c); k > 0; --k) left &= left - 1;
    write_pick(r, row, x.index(round, __ffs(left) - 1), s.conf, s.prob);
  }
}

// fp32: a read for the largest logit, one for the bins' counts and weights, and
// one for each border whose bin has more than one token, or that is drawn from:
// the bin's tokens are listed, told apart by their next eight bits, and those of
// one such value by comparing them all.  Bound by the second read: all in all 96
// vector instructions a logit (the 64-bit exponential), at four cycles each 75% of
// the SIMDs' on the CUs that have a row; the LDS works in 26%.  67 rows of 50021 44 us.
constexpr int kListed = 1024;
struct BinsF32 {
  Bins b;
  u64 mass[kBins];
  Border border;
  uint32_t sub_c[256];
  u64 sub_m[256];
  uint32_t list_n, list_min, list_max, few_n;
  uint32_t list_key[kListed];
  int list_at[kListed];
  int few[kListed];  // list entries of the border's eight bits
  uint32_t key;      // the border's value
  int seg[512];
};
__global__ __launch_bounds__(kMaxThreads) void sample_f32_kernel(SampleRows r) {
  __shared__ union {
    BinsF32 f;
    Any any;
  } sh;
  BinsF32& s = sh.f;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const Pieces<float> x((const float*)r.x + row * r.ld, r.n);
  const Settings set = settings_of(r, row);
  clear(s.b);
  for (int i = threadIdx.x; i < kBins; i += (int)blockDim.x) s.mass[i] = 0;
  float m = -INFINITY;
  uint32_t flags = 0;
  auto zero = [](uint32_t bits) { return (bits << 1) == 0; };
  auto offset = [](uint32_t bits) { return (int)((bits >> 16) & 0x7FFFu) - kLow; };  // negative: the bin of zeros
  x.each_long([&](int, const u32x4& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m = fmaxf(m, __uint_as_float(v[j]));
      if (offset(v[j]) >= kRange) flags |= outside(v[j]);
    }
  });
  m = wave_max(m);
  __syncthreads();
  if (lane == 0) s.b.part_f[wave] = m;
  if (flags) atomicOr(&s.b.flags, flags);
  __syncthreads();
  for (int w = 0; w < waves; ++w) m = fmaxf(m, s.b.part_f[w]);
  if (!by_bins(s.b.flags, m, set.scale, r.conf != nullptr)) {
    __syncthreads();
    sample_any<float>(sh.any, r, row);
    return;
  }
  auto weight = [&](uint32_t bits) { return exp_down(s.b.table, (double)__uint_as_float(bits) - (double)m, set.scale); };
  u64 high = 0;
  double soft = 0.0;
  const bool same_scale = set.scale == kScaleOne;
  x.each_long([&](int round, const u32x4& v) {
    if (x.index(round, 0) >= r.n) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int off = offset(v[j]);
      if (off >= kRange) continue;
      const int bin = off < 0 ? kRange : (int)(v[j] >> 31) * (kRange + 1) + off;  // its place
      const double w = weight(v[j]);
      const u64 units = units_of(w);
      atomicAdd(&s.b.count[bin], 1u);
      if (units) atomicAdd(&s.mass[bin], units);
      if (set.min_p > 0.0 && w >= set.min_p) high += units;
      if (r.conf) soft += same_scale ? w : exp_down(s.b.table, (double)__uint_as_float(v[j]) - (double)m, kScaleOne);
    }
  });
  __syncthreads();
#pragma unroll 1
  for (int g = wave; g < kGroups; g += waves) {
    const int b0 = place_of(g * 128 + 2 * lane), b1 = place_of(g * 128 + 2 * lane + 1);
    const uint32_t c = s.b.count[b0] + s.b.count[b1];
    if (!__ballot(c != 0)) continue;
    const u64 mt = wave_total(s.mass[b0] + s.mass[b1]);
    const uint32_t ct = wave_total(c);
    if (lane == 0) {
      s.b.group_c[g] = ct;
      s.b.group_m[g] = mt;
    }
  }
  gather_sums(s.b, high, soft);
  u64 all = 0;
  uint32_t valid = 0;
  for (int g = lane; g < 128; g += 64) {
    all += s.b.group_m[g];
    valid += s.b.group_c[g];
  }
  all = wave_total(all);
  valid = wave_total(valid);
  if (!(set.min_p > 0.0)) high = all;

  // entry `at` of the list is the border's only token, or -1: list_n tokens of
  // the value `key`
  int only = -1;
  const Draw d = draw_by(set, all, high, valid, [&](int cut, uint32_t want_c, u64 want_m) -> Border {
    __syncthreads();  // every wave has read the last cut's border, its list and its counts
    if (wave == 0) {
      const Border f = find_bin(s.b, cut != 0, want_c, want_m, [&](int bin) { return s.mass[place_of(bin)]; });
      if (lane == 0) s.border = f;
    }
    if (threadIdx.x < 256) {
      s.sub_c[threadIdx.x] = 0;
      s.sub_m[threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) {
      s.list_n = s.few_n = 0;
      s.list_min = ~0u;
      s.list_max = 0;
    }
    __syncthreads();
    Border f = s.border;
    const int bin = f.at;
    if (f.in_c == 1 && cut < 2) return f;
    const uint32_t upper = half_of_bin(bin);
    x.each_long([&](int round, const u32x4& v) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (bin == kRange ? offset(v[j]) < 0 : v[j] >> 16 == upper) {
          const uint32_t at = atomicAdd(&s.list_n, 1u), key = zero(v[j]) ? 0u : v[j];
          atomicMin(&s.list_min, key);
          atomicMax(&s.list_max, key);
          if (at < kListed) {
            s.list_key[at] = key;
            s.list_at[at] = x.index(round, j);
          }
        }
    });
    __syncthreads();
    const int n = (int)s.list_n;
    only = -1;
    if (s.list_min == s.list_max) {  // equal tokens
      if (threadIdx.x == 0) s.key = s.list_min;
      __syncthreads();
      return f;
    }
    if (n > kListed || bin == kRange) return Border{0, 0, 0, 0, 0};  // not found this way
    const uint32_t turn = bin < kRange ? 255u : 0u;  // the largest value first
    const int t = threadIdx.x;
    const uint32_t mine = t < n ? s.list_key[t] : 0;
    const int sub = ((mine >> 8) & 255u) ^ turn;
    const u64 own = t < n ? units_of(weight(mine)) : 0;
    if (t < n) {
      atomicAdd(&s.sub_c[sub], 1u);
      atomicAdd(&s.sub_m[sub], own);
    }
    __syncthreads();
    if (wave == 0) {
      const Border g = find_entry<4>(cut != 0, want_c, want_m, f.before_c, f.before_m, [&](int i) { return s.sub_c[i]; },
                                     [&](int i) { return s.sub_m[i]; });
      if (lane == 0) s.border = g;
    }
    __syncthreads();
    f = s.border;
    const bool close = t < n && sub == f.at;
    if (close) s.few[atomicAdd(&s.few_n, 1u)] = t;
    __syncthreads();
    if (close) {
      // the tokens before this one, and their weight; equal ones by index
      uint32_t bc = f.before_c;
      u64 bm = f.before_m;
      const int at = s.list_at[t];
      for (int i = 0; i < (int)s.few_n; ++i) {
        const int o = s.few[i];
        const uint32_t k = s.list_key[o];
        if (k == mine ? s.list_at[o] < at : (turn ? k > mine : k < mine)) {
          ++bc;
          bm += k == mine ? own : units_of(weight(k));
        }
      }
      if (cut != 0 ? bm < want_m && want_m <= bm + own : bc < want_c && want_c <= bc + 1) {
        s.border = {t, bc, 1, bm, own};
        s.key = mine;
      }
    }
    __syncthreads();
    f = s.border;
    only = f.at;
    return f;
  });
  if (d.at.in_c == 0) {
    __syncthreads();
    sample_any<float>(sh.any, r, row);
    return;
  }
  const double conf = exp_down(s.b.table, (double)__uint_as_float(s.key) - (double)m, kScaleOne) / soft;
  if (only >= 0) {
    if (threadIdx.x == 0) write_pick(r, row, s.list_at[only], conf, d.prob);
    return;
  }
  const int n = (int)s.list_n;
  if (n <= kListed) {  // the nth of the listed ones by index
    if ((int)threadIdx.x < n) {
      const int mine = s.list_at[threadIdx.x];
      uint32_t before = 0;
      for (int i = 0; i < n; ++i) before += s.list_at[i] < mine;
      if (before == d.nth) write_pick(r, row, mine, conf, d.prob);
    }
    return;
  }
  // more of them than are listed: by segments of 1024 tokens
  const uint32_t key = s.key;
  uint32_t nth = d.nth;
  const int seg = (r.n + 1023) / 1024;
  for (int i = threadIdx.x; i < seg; i += (int)blockDim.x) s.seg[i] = 0;
  __syncthreads();
  auto same_as = [&](uint32_t bits) { return bits == key || (key == 0 && zero(bits)); };
  x.each_long([&](int round, const u32x4& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (same_as(v[j])) atomicAdd(&s.seg[x.index(round, j) >> 10], 1);
  });
  __syncthreads();
  int at = 0;
  while (at + 1 < seg && nth >= (uint32_t)s.seg[at]) nth -= s.seg[at++];
  if (wave == 0) {
#pragma unroll 1
    for (int i0 = at * 1024; i0 < min(r.n, at * 1024 + 1024); i0 += 64) {
      const bool same = i0 + lane < r.n && same_as(__float_as_uint(x.x[i0 + lane]));
      const u64 all_same = __ballot(same);
      if (same && (uint32_t)__popcll(all_same & ((1ull << lane) - 1)) == nth) write_pick(r, row, i0 + lane, conf, d.prob);
      if (nth < (uint32_t)__popcll(all_same)) break;
      nth -= __popcll(all_same);
    }
  }
}

}  // namespace

hipError_t launch_sample_commit(acache_dtype dt, const SampleRows& r, int rows, hipStream_t s) {
  // bf16: with a row for every CU at most, 1024 threads for each (rows of 126464:
  // one 21.4 us, 24.0 with 512; 256 26.3, 30.2); with more, four rows side by side
  // on a CU, 512 threads and 64 registers each, so that one row's search runs
  // behind the others' reads (512 rows 44.6, 50.9 with 1024 threads; 1024 77, 99)
  if (dt == ACACHE_F32) hipLaunchKernelGGL(sample_f32_kernel, dim3(rows), dim3(kMaxThreads), 0, s, r);
  else if (rows <= 256) hipLaunchKernelGGL((sample_bf16_kernel<kMaxThreads, 4>), dim3(rows), dim3(kMaxThreads), 0, s, r);
  else hipLaunchKernelGGL((sample_bf16_kernel<512, 8>), dim3(rows), dim3(512), 0, s, r);
  return hipGetLastError();
}

}  // namespace acache
