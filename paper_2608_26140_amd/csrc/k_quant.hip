// Storing rows into the 8-bit KV cache and reading rows back (gfx950).
#include <algorithm>

#include "internal.h"
#include "quant.h"

namespace acache {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;

constexpr int kThreads = 256;
constexpr int kMaxBlock = 256;  // slots that share a scale, at most

// Eight consecutive elements as they lie in memory; none: zeros.
template <typename T>
struct Piece;
template <>
struct Piece<bf16> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void none() { w = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ float at(int j) const {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
  }
  // the largest magnitude, infinities and NaN above all (their bits are), two
  // elements at a time
  __device__ __forceinline__ float top() const {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[j] & 0x7FFF7FFFu));
    return __uint_as_float((uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16);
  }
  // codes of finite elements within the scale's range
  __device__ __forceinline__ u32x2 encode(float scale) const {
    u32x2 c;
#pragma unroll
    for (int j = 0; j < 2; ++j) c[j] = pair(w[2 * j], scale) | pair(w[2 * j + 1], scale) << 16;
    return c;
  }
  // two codes in the low half (the form that writes the high half of what is
  // there is not used: the compiler gives it the first form's operand)
  static __device__ __forceinline__ uint32_t pair(uint32_t x, float scale) {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const i16x2 none = {0, 0};
    return __builtin_bit_cast(
        uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(none, __builtin_bit_cast(bf16x2, x), scale, false));
  }
};
template <>
struct Piece<float> {
  f32x4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = reinterpret_cast<const f32x4*>(p)[0];
    v[1] = reinterpret_cast<const f32x4*>(p)[1];
  }
  __device__ __forceinline__ void none() { v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float at(int j) const { return v[j >> 2][j & 3]; }
  __device__ __forceinline__ float top() const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(at(j)) & 0x7FFFFFFFu);
    return __uint_as_float(m);
  }
  __device__ __forceinline__ u32x2 encode(float scale) const {
    const float inv = pow2_byte(254 - (int)(__float_as_uint(scale) >> 23));
    return u32x2{encode4(v[0][0] * inv, v[0][1] * inv, v[0][2] * inv, v[0][3] * inv),
                 encode4(v[1][0] * inv, v[1][1] * inv, v[1][2] * inv, v[1][3] * inv)};
  }
};
// The largest finite magnitude, and codes of any elements.
template <typename T>
__device__ __forceinline__ float finite_top(const Piece<T>& x) {
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(x.at(j)) < INFINITY ? fabsf(x.at(j)) : 0.f);
  return m;
}
template <typename T>
__device__ __forceinline__ u32x2 encode_any(const Piece<T>& x, float inv) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = code_arg(x.at(j), inv);
  return u32x2{encode4(y[0], y[1], y[2], y[3]), encode4(y[4], y[5], y[6], y[7])};
}

// Maximum of non-negative bit patterns (infinities and NaN above all) over the
// workgroup.
__device__ __forceinline__ float group_top(float m, uint32_t* red) {
  uint32_t u = __float_as_uint(m);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) u = max(u, (uint32_t)__shfl_xor((int)u, o));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = u;
  __syncthreads();
  return __uint_as_float(max(max(red[0], red[1]), max(red[2], red[3])));
}

// ============================================================================
// Store.  A block is quantised by the workgroups of one of its rows, the last
// that names one of its slots, one workgroup for each KV head and for K and V:
// the maximum over the new rows, the scale, the codes, and the entries that
// stay.  The rows of a call may name slots in any order, so a block's rows are
// found through a map from its slots to the last row of each.
//   Up to kSmallRows rows every workgroup reads all the call's slots and makes
// its block's map in LDS: one launch.  (One launch against two, us a call, warm:
// 32 rows 7.2 / 9.1, 1024 rows of 32 heads 10.5 / 11.7 and of 4 heads 8.2 / 9.7;
// 2048 rows 19.4 / 17.7 and 9.4 / 10.0, 4096 rows 36.9 / 25.3 and 12.1 / 10.6.
// They cross near 1600 rows of 32 heads and 2700 of 4.)
//   Beyond, a launch of its own leaves the map in the workspace.  Entries of
// slots that are not named stay what they were: the launch that quantises takes
// an entry for a row of this call only where that row's slot is the entry's
// own, which no stale entry can pretend.
// Bound by HBM: 3 bytes an element of bf16.  Workgroups of neighbouring heads
// are neighbours in the grid, so that whole rows are read and written together
// (8192 rows of 32 heads of 128, from cold caches: 43 us, 4.6 TB/s, and 4.8 the
// map; with a head's workgroups together 85 in all).  A small call is its chain
// of reads: slots, rows and old scale, codes (32 rows of 32 heads: 7.2 us).
// ============================================================================
constexpr int kSmallRows = 1024;

template <typename T>
struct StoreArgs {
  const T* src[2];       // K, V rows [n, src_ld]
  uint8_t* codes[2];     // [n_slots, ld]
  float* scales[2];      // [blocks, heads]
  int64_t src_ld, ld, n_slots;
  const int32_t* slots;  // [n]
  const int32_t* row_of;
  const int32_t* last_of;
  int n, heads, head_dim, shift;
};

// The last row of a run of rows in one block: a block's last row is one.  A row
// without a slot ends a run too, also where its slot number lies in the short
// last block.
__device__ __forceinline__ bool ends_run(const int32_t* slots, int i, int n, int64_t n_slots, int shift) {
  return i + 1 == n || slots[i + 1] >= n_slots || (slots[i + 1] >> shift) != (slots[i] >> shift);
}

// Leaves the last row of every slot that a call names, and of every block, in
// tables of any earlier contents.  A row puts itself into its entry; where it
// takes out another row of this call it offers that row to the entry again, as
// a maximum.  Whoever takes the last row out puts it back, so it stays.  (Two
// launches, one that clears the entries and one that raises them, took 9.5 us
// for 8192 rows where this takes 4.6.)  64 rows at one entry of last_of would
// queue for it, so only the ends of runs of rows of one block go there.
template <typename F>
__device__ __forceinline__ void keep_last(int32_t* entry, int i, F is_row) {
  const int other = atomicExch(entry, i);
  if (other != i && is_row(other)) atomicMax(entry, other);
}
__global__ __launch_bounds__(kThreads) void quant_map_kernel(const int32_t* __restrict__ slots, int n, int64_t n_slots,
                                                             int shift, int32_t* __restrict__ row_of,
                                                             int32_t* __restrict__ last_of) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (at >= n) return;
  const int i = (int)at, s = slots[i];
  if (s < 0 || s >= n_slots) return;
  keep_last(row_of + s, i, [&](int j) { return j >= 0 && j < n && slots[j] == s; });
  // a stale entry may name a row whose slot number lies in the short last block
  // past its end: that row is stored nowhere and must not stand for the block
  if (ends_run(slots, i, n, n_slots, shift))
    keep_last(last_of + (s >> shift), i,
              [&](int j) { return j >= 0 && j < n && slots[j] < n_slots && slots[j] >> shift == s >> shift; });
}

// Quantises one block and head from its map win (LDS): the row stored at each
// slot, -1 where none is.  IT: 8-element pieces of the block for each thread.
template <typename T, int IT>
__device__ __forceinline__ void store_block(const StoreArgs<T>& a, int which, int g, int blk, const int32_t* win,
                                            uint32_t* red, bool missing) {
  const int tid = threadIdx.x;
  const int64_t first = (int64_t)blk << a.shift;
  // pieces tid, tid + kThreads, ..: piece c of the block's row r
  const int chunks = a.head_dim >> 3, rows = 1 << a.shift;
  const int dr = kThreads / chunks, dc = kThreads - dr * chunks, r0 = tid / chunks, c0 = tid - r0 * chunks;
  auto next = [&](int& r, int& c) {
    r += dr;
    c += dc;
    if (c >= chunks) {
      c -= chunks;
      ++r;
    }
  };
  const T* src = a.src[which] + g * a.head_dim;
  uint8_t* codes = a.codes[which] + g * a.head_dim;
  float* sp = a.scales[which] + (int64_t)blk * a.heads + g;
  const float old = *sp;
  Piece<T> v[IT];
  float mx = 0.f;
  int r = r0, c = c0;
#pragma unroll
  for (int it = 0; it < IT; ++it, next(r, c)) {
    const int w = r < rows ? win[r] : -1;
    if (w >= 0) v[it].load(src + (int64_t)w * a.src_ld + c * 8);
    else v[it].none();
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) mx = __uint_as_float(max(__float_as_uint(mx), __float_as_uint(v[it].top())));
  mx = group_top(mx, red);
  // an element that is not finite, or past the largest scale's range: the
  // careful way, which no ordinary block takes
  const bool odd = !(mx <= kMaxCode * pow2_byte(kMaxScaleByte));
  if (odd) {
    mx = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it) mx = fmaxf(mx, finite_top(v[it]));
    __syncthreads();
    mx = group_top(mx, red);
  }
  const int was = old > 0.f ? (int)(__float_as_uint(old) >> 23) : 0;
  int e = scale_byte(mx);
  if (missing && was) e = max(e, min(was, kMaxScaleByte));
  r = r0;
  c = c0;
#pragma unroll
  for (int it = 0; it < IT; ++it, next(r, c)) {
    if (r >= rows || first + r >= a.n_slots) continue;
    uint8_t* p = codes + (first + r) * a.ld + c * 8;
    if (win[r] >= 0) {
      *reinterpret_cast<u32x2*>(p) = odd ? encode_any(v[it], pow2_byte(254 - e)) : v[it].encode(pow2_byte(e));
    } else if (!was) {
      *reinterpret_cast<u32x2*>(p) = u32x2{0u, 0u};  // of an empty block: reads as zero before and after
    } else if (e > was) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
      float lo[4], hi[4];
      decode4(w[0], lo);
      decode4(w[1], hi);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = __builtin_amdgcn_ldexpf(lo[j], was - e);
        hi[j] = __builtin_amdgcn_ldexpf(hi[j], was - e);
      }
      *reinterpret_cast<u32x2*>(p) = u32x2{encode4(lo[0], lo[1], lo[2], lo[3]), encode4(hi[0], hi[1], hi[2], hi[3])};
    }
  }
  if (tid == 0) *sp = pow2_byte(e);  // every thread read the old scale ahead of the barrier
}

template <typename T, int IT, bool SMALL>
__global__ __launch_bounds__(kThreads) void quant_store_kernel(StoreArgs<T> a) {
  __shared__ int32_t all[SMALL ? kSmallRows : 1];  // the call's slots, -1 those that are not there
  __shared__ int32_t win[kMaxBlock];
  __shared__ int32_t found[kMaxBlock];  // rows of this workgroup's that may be their block's last
  __shared__ int n_found;
  __shared__ uint32_t red[kThreads / 64];
  const int tid = threadIdx.x, block = 1 << a.shift;
  const unsigned chunk = blockIdx.x / (2u * a.heads), h = blockIdx.x - chunk * (2u * a.heads);
  const int which = (int)h >= a.heads, g = (int)h - which * a.heads;
  const int i0 = (int)chunk << a.shift;
  if (tid == 0) n_found = 0;
  if constexpr (SMALL) {
    for (int i = tid; i < a.n; i += kThreads) {
      const int s = a.slots[i];
      all[i] = s >= 0 && s < a.n_slots ? s : -1;
    }
  }
  __syncthreads();
  if (tid < block && tid < a.n - i0) {
    if constexpr (SMALL) {
      if (all[i0 + tid] >= 0 && ends_run(all, i0 + tid, a.n, a.n_slots, a.shift)) found[atomicAdd(&n_found, 1)] = i0 + tid;
    } else {
      const int s = a.slots[i0 + tid];
      if (s >= 0 && s < a.n_slots && a.last_of[s >> a.shift] == i0 + tid) found[atomicAdd(&n_found, 1)] = s >> a.shift;
    }
  }
  __syncthreads();
  for (int o = 0; o < n_found; ++o) {
    int blk = found[o];
    if constexpr (SMALL) {
      const int row = blk;
      blk = all[row] >> a.shift;
      int later = 0;
      for (int i = row + 1 + tid; i < a.n; i += kThreads) later |= all[i] >= 0 && all[i] >> a.shift == blk;
      if (__syncthreads_or(later)) continue;
    }
    if (tid < block) {
      win[tid] = -1;
      const int64_t s = ((int64_t)blk << a.shift) + tid;
      if (!SMALL && s < a.n_slots) {
        const int c = a.row_of[s];
        if (c >= 0 && c < a.n && a.slots[c] == s) win[tid] = c;
      }
    }
    __syncthreads();
    if constexpr (SMALL) {
      for (int i = tid; i < a.n; i += kThreads)
        if (all[i] >= 0 && all[i] >> a.shift == blk) atomicMax(win + (all[i] & (block - 1)), i);
      __syncthreads();
    }
    const int64_t s = ((int64_t)blk << a.shift) + tid;
    const bool missing = __syncthreads_or(tid < block && s < a.n_slots && win[tid] < 0);
    store_block<T, IT>(a, which, g, blk, win, red, missing);
    __syncthreads();  // win and red are free
  }
}

// ============================================================================
// Load: value = code * scale, exact.  One thread per 16 codes of K or V, 16
// bytes read and 32 written (bf16).  Bound by HBM: 8192 rows of 32 heads of 128
// take 44 us from cold caches, 4.6 TB/s.
// ============================================================================
template <typename T>
__global__ __launch_bounds__(kThreads) void quant_load_kernel(const uint8_t* __restrict__ kc,
                                                              const uint8_t* __restrict__ vc,
                                                              const float* __restrict__ ks,
                                                              const float* __restrict__ vs, int64_t ld,
                                                              int64_t n_slots, int shift, int heads, int head_dim,
                                                              const int32_t* __restrict__ slots, int n,
                                                              T* __restrict__ kd, T* __restrict__ vd, int64_t dst_ld) {
  const int per_head = head_dim >> 4, chunks = heads * per_head;
  const bool is_v = blockIdx.y != 0;
  const uint8_t* codes = is_v ? vc : kc;
  const float* scales = is_v ? vs : ks;
  T* dst = is_v ? vd : kd;
  if (!dst) return;
  for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < (int64_t)n * chunks;
       at += (int64_t)gridDim.x * kThreads) {
    const int i = (int)(at / chunks), c = (int)(at - (int64_t)i * chunks);
    const int s = slots[i];
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = 0.f;
    if (s >= 0 && s < n_slots) {
      const float sc = pow2_below(scales[(int64_t)(s >> shift) * heads + c / per_head]);
      if (sc > 0.f) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(codes + (int64_t)s * ld + c * 16);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float d[4];
          decode4(w[q], d);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * q + j] = d[j] * sc;
        }
      }
    }
    T* p = dst + (int64_t)i * dst_ld + c * 16;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        bf16x8 w;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = (bf16)v[8 * q + j];
        reinterpret_cast<bf16x8*>(p)[q] = w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        reinterpret_cast<f32x4*>(p)[q] = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    }
  }
}

__global__ __launch_bounds__(kThreads) void iota_kernel(int32_t* out, int n) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) out[i] = (int32_t)i;
}

template <typename T, bool SMALL>
void store_items(const StoreArgs<T>& a, hipStream_t s) {
  const dim3 grid((unsigned)((((int64_t)a.n + (1 << a.shift) - 1) >> a.shift) * 2 * a.heads));
  const int items = (a.head_dim >> 3) << a.shift;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a); };
  if (items <= kThreads) go(quant_store_kernel<T, 1, SMALL>);
  else if (items <= 2 * kThreads) go(quant_store_kernel<T, 2, SMALL>);
  else if (items <= 4 * kThreads) go(quant_store_kernel<T, 4, SMALL>);
  else if (items <= 8 * kThreads) go(quant_store_kernel<T, 8, SMALL>);
  else go(quant_store_kernel<T, 16, SMALL>);
}

template <typename T>
hipError_t store(const QuantPool& p, const void* k, const void* v, int64_t src_ld, int n, const int32_t* slots,
                 int32_t* map, hipStream_t s) {
  StoreArgs<T> a;
  a.src[0] = (const T*)k;
  a.src[1] = (const T*)v;
  for (int i = 0; i < 2; ++i) {
    a.codes[i] = (uint8_t*)p.codes[i];
    a.scales[i] = p.scales[i];
  }
  a.src_ld = src_ld;
  a.ld = p.ld;
  a.n_slots = p.n_slots;
  a.slots = slots;
  int32_t* row_of = map;
  int32_t* last_of = map + p.n_slots;
  a.row_of = row_of;
  a.last_of = last_of;
  a.n = n;
  a.heads = p.heads;
  a.head_dim = p.head_dim;
  a.shift = p.shift;
  if (n <= kSmallRows) {
    store_items<T, true>(a, s);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(quant_map_kernel, dim3((unsigned)(((int64_t)n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                     slots, n, p.n_slots, p.shift, row_of, last_of);
  store_items<T, false>(a, s);
  return hipGetLastError();
}

}  // namespace

size_t quant_map_bytes(int64_t n_slots, int shift) {
  return (size_t)(n_slots + ((n_slots + (1 << shift) - 1) >> shift)) * sizeof(int32_t);
}

hipError_t launch_iota(int32_t* out, int n, hipStream_t s) {
  hipLaunchKernelGGL(iota_kernel, dim3((unsigned)(((int64_t)n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, out, n);
  return hipGetLastError();
}

hipError_t launch_quant_store(acache_dtype dt, const QuantPool& p, const void* k, const void* v, int64_t src_ld, int n,
                              const int32_t* slots, int32_t* map, hipStream_t s) {
  return dt == ACACHE_BF16 ? store<bf16>(p, k, v, src_ld, n, slots, map, s)
                           : store<float>(p, k, v, src_ld, n, slots, map, s);
}

hipError_t launch_quant_load(acache_dtype dt, const QuantPool& p, const int32_t* slots, int n, void* k, void* v,
                             int64_t dst_ld, hipStream_t s) {
  const int64_t work = (int64_t)n * p.heads * (p.head_dim >> 4);
  const dim3 grid((unsigned)std::min<int64_t>((work + kThreads - 1) / kThreads, 1 << 20), 2);
  auto go = [&](auto kernel, auto* kd, auto* vd) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, (const uint8_t*)p.codes[0], (const uint8_t*)p.codes[1],
                       (const float*)p.scales[0], (const float*)p.scales[1], p.ld, p.n_slots, p.shift, p.heads,
                       p.head_dim, slots, n, kd, vd, dst_ld);
  };
  if (dt == ACACHE_BF16) go(quant_load_kernel<bf16>, (bf16*)k, (bf16*)v);
  else go(quant_load_kernel<float>, (float*)k, (float*)v);
  return hipGetLastError();
}

}  // namespace acache
