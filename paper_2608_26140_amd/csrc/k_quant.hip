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

__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
  const bf16x8 w = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p));
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)w[j];
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = a[j];
    v[4 + j] = b[j];
  }
}

// ============================================================================
// Store.  The rows of a call may name slots in any order, so a block's new
// rows are found through a map from slots to rows in the workspace: one
// launch marks the slots that are named (the entries of the others stay what
// they were), the next leaves the highest row of each, and the one that
// quantises takes an entry for a row of this call only where that row's slot
// is the entry's own, which no stale entry can pretend.  A block is quantised
// by the workgroups of one of its rows (its highest), one for each KV head
// and for K and V: the maximum over the new rows, the scale, the codes, and
// the entries that stay.
// ============================================================================
__global__ __launch_bounds__(kThreads) void quant_clear_kernel(const int32_t* __restrict__ slots, int n,
                                                               int64_t n_slots, int shift, int32_t* __restrict__ row_of,
                                                               int32_t* __restrict__ last_of) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int s = slots[i];
  if (s < 0 || s >= n_slots) return;
  row_of[s] = -1;
  last_of[s >> shift] = -1;
}
__global__ __launch_bounds__(kThreads) void quant_map_kernel(const int32_t* __restrict__ slots, int n, int64_t n_slots,
                                                             int shift, int32_t* __restrict__ row_of,
                                                             int32_t* __restrict__ last_of) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int s = slots[i];
  if (s < 0 || s >= n_slots) return;
  atomicMax(row_of + s, i);
  atomicMax(last_of + (s >> shift), i);
}

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

// IT: 8-element pieces of a block and head for each thread.
template <typename T, int IT>
__global__ __launch_bounds__(kThreads) void quant_store_kernel(StoreArgs<T> a) {
  __shared__ int32_t win[kMaxBlock];   // the row stored at each slot of the block, -1: none
  __shared__ int32_t owned[kMaxBlock];
  __shared__ int n_owned;
  __shared__ float red[kThreads / 64];
  __shared__ int missing;
  const int tid = threadIdx.x, block = 1 << a.shift;
  const int which = (int)blockIdx.y >= a.heads, g = blockIdx.y - which * a.heads;
  if (tid == 0) n_owned = 0;
  __syncthreads();
  const int i0 = blockIdx.x << a.shift;
  if (tid < block && tid < a.n - i0) {
    const int s = a.slots[i0 + tid];
    if (s >= 0 && s < a.n_slots && a.last_of[s >> a.shift] == i0 + tid) owned[atomicAdd(&n_owned, 1)] = s >> a.shift;
  }
  __syncthreads();
  const int chunks = a.head_dim >> 3, items = chunks << a.shift;
  const T* src = a.src[which] + g * a.head_dim;
  uint8_t* codes = a.codes[which] + g * a.head_dim;
  for (int o = 0; o < n_owned; ++o) {
    const int blk = owned[o];
    const int64_t first = (int64_t)blk << a.shift;
    if (tid == 0) missing = 0;
    __syncthreads();
    if (tid < block) {
      const int64_t s = first + tid;
      int w = -1;
      if (s < a.n_slots) {
        const int c = a.row_of[s];
        if (c >= 0 && c < a.n && a.slots[c] == s) w = c;
        if (w < 0) missing = 1;
      }
      win[tid] = w;
    }
    __syncthreads();
    float v[IT][8];
    float mx = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int item = it * kThreads + tid, r = item / chunks, c = item - r * chunks;
      const int w = item < items ? win[r] : -1;
      if (w >= 0) {
        load8(src + (int64_t)w * a.src_ld + c * 8, v[it]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[it][j] = 0.f;
      }
    }
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int j = 0; j < 8; ++j) mx = fmaxf(mx, fabsf(v[it][j]) < INFINITY ? fabsf(v[it][j]) : 0.f);
    mx = wave_max(mx);
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float* sp = a.scales[which] + (int64_t)blk * a.heads + g;
    const float old = *sp;
    const int was = old > 0.f ? (int)(__float_as_uint(old) >> 23) : 0;
    int e = scale_byte(mx);
    if (missing && was) e = max(e, min(was, kMaxScaleByte));
    const float inv = pow2_byte(254 - e);
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int item = it * kThreads + tid, r = item / chunks, c = item - r * chunks;
      if (item >= items || first + r >= a.n_slots) continue;
      uint8_t* p = codes + (first + r) * a.ld + c * 8;
      if (win[r] >= 0) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = code_arg(v[it][j], inv);
        *reinterpret_cast<u32x2*>(p) = u32x2{encode4(y[0], y[1], y[2], y[3]), encode4(y[4], y[5], y[6], y[7])};
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
    __syncthreads();  // every thread has read the old scale, win and red
    if (tid == 0) *sp = pow2_byte(e);
  }
}

// ============================================================================
// Load: one thread per 16 codes of K or V.
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
      const float sc = scales[(int64_t)(s >> shift) * heads + c / per_head];
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

template <typename T>
void store_items(const StoreArgs<T>& a, dim3 grid, int it, hipStream_t s) {
  switch (it) {
    case 1: hipLaunchKernelGGL((quant_store_kernel<T, 1>), grid, dim3(kThreads), 0, s, a); break;
    case 2: hipLaunchKernelGGL((quant_store_kernel<T, 2>), grid, dim3(kThreads), 0, s, a); break;
    case 4: hipLaunchKernelGGL((quant_store_kernel<T, 4>), grid, dim3(kThreads), 0, s, a); break;
    case 8: hipLaunchKernelGGL((quant_store_kernel<T, 8>), grid, dim3(kThreads), 0, s, a); break;
    default: hipLaunchKernelGGL((quant_store_kernel<T, 16>), grid, dim3(kThreads), 0, s, a); break;
  }
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
  const unsigned wgs = (unsigned)((n + kThreads - 1) / kThreads);
  hipLaunchKernelGGL(quant_clear_kernel, dim3(wgs), dim3(kThreads), 0, s, slots, n, p.n_slots, p.shift, row_of, last_of);
  hipLaunchKernelGGL(quant_map_kernel, dim3(wgs), dim3(kThreads), 0, s, slots, n, p.n_slots, p.shift, row_of, last_of);
  const int need = (((p.head_dim >> 3) << p.shift) + kThreads - 1) / kThreads;
  int it = 1;
  while (it < need) it *= 2;
  store_items(a, dim3((unsigned)((n + (1 << p.shift) - 1) >> p.shift), (unsigned)(2 * p.heads)), it, s);
  return hipGetLastError();
}

}  // namespace

size_t quant_map_bytes(int64_t n_slots, int shift) {
  return (size_t)(n_slots + ((n_slots + (1 << shift) - 1) >> shift)) * sizeof(int32_t);
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
