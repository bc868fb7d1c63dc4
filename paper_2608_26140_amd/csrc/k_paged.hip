// A cache in blocks with a table of block ids for each request: rotating and
// storing new rows, and attention of a step's rows over a request's positions.
//
// Position p of request b is slot tables[b][p / block] * block + p % block.  A
// position past the table, or whose entry names no block of the pools, has no
// slot: nothing is stored there, and it reads as a key and a value of zeros.
#include <algorithm>

#include "device.h"
#include "internal.h"

namespace acache {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

// Slot of a request's position, -1 if it has none.
__device__ __forceinline__ int slot_of(const PagedCache& c, const int32_t* __restrict__ table, int at) {
  const uint32_t blk = (uint32_t)at / (uint32_t)c.block;
  if (at < 0 || blk >= (uint32_t)c.max_blocks) return -1;
  const int id = table[blk];
  return id < 0 || id >= c.n_blocks ? -1 : id * c.block + (int)((uint32_t)at - blk * (uint32_t)c.block);
}

// ---------------------------------------------------------------- append
template <typename T, int V>
struct Run {  // V consecutive elements of one half of a head
  T e[V];
};

// Rows of K and Q are turned by pos * theta_i, theta_i = base^(-2i/d), in each
// half-split pair (i, i + d/2); rows of V are copied.  An item is V pairs of
// one head: two runs of V elements, in and out.  A workgroup takes `rows` rows
// and the items [blockIdx.y, + gridDim.y, ..) of each; it evaluates every
// angle of its rows once (fp64, rotary_sincos) into LDS while its first items
// are on their way.  Bound by memory: each element is read and written once.
template <typename T, int V>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedCache c, AppendRows r, int rows, double log2_base) {
  extern __shared__ float2 turn[];  // [rows][half]: cos, sin
  const int half = c.head_dim >> 1, per_head = half / V;
  const int heads = (r.q ? r.heads : 0) + 2 * c.kv_heads;
  const int items = heads * per_head;
  const int first = blockIdx.x * rows;
  const int here = min(rows, r.n - first);
  for (int t = threadIdx.x; t < here * half; t += 256) {
    const int row = t / half, i = t - row * half;
    float sn = 0.f, cs = 0.f;
    rotary_sincos((double)r.pos[first + row] * exp2(-(2.0 * i / c.head_dim) * log2_base), &sn, &cs);
    turn[t] = make_float2(cs, sn);
  }
  __syncthreads();
  for (int row = 0; row < here; ++row) {
    const int m = first + row, b = m / r.per_request, pos = r.pos[m];
    const int64_t slot = pos < 0 ? -1 : slot_of(c, c.tables + (int64_t)b * c.table_ld, r.at ? r.at[m] : pos);
    for (int t = blockIdx.y * 256 + threadIdx.x; t < items; t += gridDim.y * 256) {
      int h = t / per_head;
      const int i = (t - h * per_head) * V;
      const T* src;
      T* dst;
      bool turned = true;
      if (h < heads - 2 * c.kv_heads) {
        src = (const T*)r.q + (int64_t)m * r.q_ld + h * c.head_dim;
        dst = (T*)r.q_out + (int64_t)m * r.q_out_ld + h * c.head_dim;
      } else {
        if (slot < 0) continue;
        h -= heads - 2 * c.kv_heads;
        turned = h < c.kv_heads;
        if (!turned) h -= c.kv_heads;
        src = turned ? (const T*)r.k + (int64_t)m * r.k_ld : (const T*)r.v + (int64_t)m * r.v_ld;
        dst = (T*)(turned ? c.k : c.v) + slot * c.ld;
        src += h * c.head_dim;
        dst += h * c.head_dim;
      }
      Run<T, V> lo, hi;
      __builtin_memcpy(&lo, src + i, sizeof(lo));
      __builtin_memcpy(&hi, src + i + half, sizeof(hi));
      if (turned) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float2 a = pos < 0 ? make_float2(0.f, 0.f) : turn[row * half + i + j];
          const float x = to_f32(lo.e[j]), y = to_f32(hi.e[j]);
          lo.e[j] = from_f32<T>(pos < 0 ? 0.f : x * a.x - y * a.y);
          hi.e[j] = from_f32<T>(pos < 0 ? 0.f : y * a.x + x * a.y);
        }
      }
      __builtin_memcpy(dst + i, &lo, sizeof(lo));
      __builtin_memcpy(dst + i + half, &hi, sizeof(hi));
    }
  }
}

// ---------------------------------------------------------------- attention
// Query p = i * rep + j of KV head g is row i of the request, head g * rep + j.
struct Group {
  int b, g, split, tile;
};

// Workgroups are dealt round-robin to the 8 XCDs: the query tiles that read the
// same keys run on one XCD, one after the other, so that its L2 serves all but
// the first.
__device__ __forceinline__ bool group_of(const PagedCache& c, const PagedPlan& p, Group& o) {
  const int id = blockIdx.x;
  int k = id / (8 * p.tiles) * 8 + (id & 7);
  o.tile = (id >> 3) % p.tiles;
  o.g = k % c.kv_heads;
  k /= c.kv_heads;
  o.split = k % p.splits;
  o.b = k / p.splits;
  return o.b < c.batch;
}

// Keys [begin, end) of a split of `len`: equal shares in whole multiples of 128
// (a step of 32 keys for each of a workgroup's waves).
__device__ __forceinline__ void share_of(int len, int splits, int split, int& begin, int& end) {
  const int per = ((len + splits - 1) / splits + 127) & ~127;
  begin = (int)min((int64_t)len, (int64_t)split * per);
  end = min(len, begin + per);
}

__device__ __forceinline__ int capped_len(const PagedCache& c, int n) {
  return (int)min((int64_t)max(n, 0), (int64_t)c.max_blocks * c.block);
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Bits set where one of the two bf16 in a word is an infinity or NaN.
__device__ __forceinline__ bool odd_word(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Attention of 16 QT queries of a KV head over a share of the keys.  Four
// waves take 32 keys each at a time and keep their own running maximum, sum
// and output; they meet at the end.  Nothing passes through LDS on the way:
//  - S^T = K Q^T on MFMA 16x16x32: a lane's K fragment is 16 consecutive bytes
//    of a key's row, straight from memory; the result leaves a lane four keys
//    (4 (lane / 16) + j) of two 16-key tiles for query lane % 16, whose maxima
//    need two exchanges between lanes;
//  - O^T = V^T P^T: those eight keys, in that order, are the lane's B fragment
//    (the order of the contraction is free), and for the A fragment a lane
//    loads 16 bytes of each of the same eight keys' rows, elements 8 (lane %
//    16) and on, and turns the 8 x 8 block in registers: row m of product i is
//    element 8 m + i.
// 16 KB are loaded a step and wave; eight waves a CU keep 128 KB in flight,
// several times what the memory's latency asks for at a CU's share of its rate.
// A weight is rounded to bf16 for its product with V (2^-8 relative at most); its sum
// is of the unrounded ones.
template <int QT>
__global__ __launch_bounds__(256) void paged_attention_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  constexpr int LDO = 132;  // padded rows of the exchange
  __shared__ float s_out[4][16][LDO];
  __shared__ float s_m[4][16], s_l[4][16];
  Group gr;
  if (!group_of(c, p, gr)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 15, lg = lane >> 4;
  const int rep = r.heads / c.kv_heads, nq = r.per_request * rep;
  const int q0 = gr.tile * 16 * QT;

  int klen[QT], longest = 0, shortest = 0x7FFFFFFF;
  bf16x8 qf[QT][4];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int q = q0 + t * 16 + ln;
    const bool real = q < nq;
    const int i = real ? q / rep : 0;
    const int64_t row = (int64_t)gr.b * r.per_request + i;
    klen[t] = real ? capped_len(c, r.key_len[row]) : 0;
    longest = max(longest, klen[t]);
    if (real) shortest = min(shortest, klen[t]);
    const bf16* src = (const bf16*)r.q + row * r.q_ld + (gr.g * rep + (real ? q - i * rep : 0)) * 128 + lg * 8;
#pragma unroll
    for (int k = 0; k < 4; ++k) qf[t][k] = *reinterpret_cast<const bf16x8*>(src + k * 32);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    longest = max(longest, __shfl_xor(longest, o));
    shortest = min(shortest, __shfl_xor(shortest, o));
  }
  longest = __builtin_amdgcn_readfirstlane(longest);
  shortest = __builtin_amdgcn_readfirstlane(shortest);

  int begin, end;
  share_of(longest, p.splits, gr.split, begin, end);
  const int32_t* table = c.tables + (int64_t)gr.b * c.table_ld;
  const bf16* kp = (const bf16*)c.k + gr.g * 128;
  const bf16* vp = (const bf16*)c.v + gr.g * 128;
  const float scale = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)

  float m[QT], l[QT];
  f32x4 acc[QT][8];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int k0 = begin + wave * 32; k0 < end; k0 += 128) {
    // the slot of key k0 + lane % 32; past the end, the last key's again
    const int mine = slot_of(c, table, min(k0 + (lane & 31), end - 1));
    u32x4 kr[2][4], vr[8];
    int ks[2], vs[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      ks[t] = __shfl(mine, t * 16 + ln);
      const bf16* src = kp + (int64_t)max(ks[t], 0) * c.ld + lg * 8;
#pragma unroll
      for (int k = 0; k < 4; ++k) kr[t][k] = *reinterpret_cast<const u32x4*>(src + k * 32);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      vs[e] = __shfl(mine, (e & 4) * 4 + lg * 4 + (e & 3));
      vr[e] = *reinterpret_cast<const u32x4*>(vp + (int64_t)max(vs[e], 0) * c.ld + ln * 8);
    }
    if (__ballot(mine < 0)) {  // keys without a slot are zeros
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (ks[t] < 0) kr[t][k] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (vs[e] < 0) vr[e] = u32x4{0, 0, 0, 0};
    }
    // An infinity or NaN of V at a key that some query does not attend to must
    // not reach it through a weight of 0: such elements are left out of the
    // product and added for the queries that do attend.
    bool odd = false;
    if (k0 + 32 > shortest) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) odd |= odd_word(vr[e][w]);
      odd = __ballot(odd) != 0;
      if (odd) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t x = vr[e][w];
            if ((x & 0x7F80u) == 0x7F80u) x &= 0xFFFF0000u;
            if ((x & 0x7F800000u) == 0x7F800000u) x &= 0xFFFFu;
            vr[e][w] = x;
          }
      }
    }
    // A fragment i: element 8 ln + i of the eight keys
    bf16x8 va[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      u32x4 even, odds;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        even[k] = __builtin_amdgcn_perm(vr[2 * k + 1][w], vr[2 * k][w], 0x05040100u);
        odds[k] = __builtin_amdgcn_perm(vr[2 * k + 1][w], vr[2 * k][w], 0x07060302u);
      }
      va[2 * w] = __builtin_bit_cast(bf16x8, even);
      va[2 * w + 1] = __builtin_bit_cast(bf16x8, odds);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) s[h] = mfma16(__builtin_bit_cast(bf16x8, kr[h][k]), qf[t][k], s[h]);
      float top = m[t];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[h][j] = k0 + h * 16 + lg * 4 + j < klen[t] ? s[h][j] * scale : -INFINITY;
          top = fmaxf(top, s[h][j]);
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__ballot(top > m[t])) {
        const float f = m[t] == top ? 1.f : __builtin_amdgcn_exp2f(m[t] - top);
        l[t] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[t][i] *= f;
        m[t] = top;
      }
      const float from = top == -INFINITY ? 0.f : top;
      bf16x8 pf;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float w = __builtin_amdgcn_exp2f(s[h][j] - from);
          s[h][j] = w;
          l[t] += w;
          pf[h * 4 + j] = (bf16)w;
        }
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[t][i] = mfma16(va[i], pf, acc[t][i]);
      if (odd) {
#pragma unroll 1
        for (int key = 0; key < 32; ++key) {
          float w = 0.f;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key >> 4 == h && (key & 3) == j) w = s[h][j];
          w = (float)(bf16)__shfl(w, (key & 12) * 4 + ln);
          const int64_t slot = __shfl(mine, key);
          const bool seen = k0 + key < klen[t] && slot >= 0;
          const bf16* src = vp + (seen ? slot * c.ld : 0) + lg * 32;
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = seen ? to_f32(src[e * 8 + i]) : 0.f;
              if (!(fabsf(v) < INFINITY)) acc[t][i][e] += w * v;
            }
        }
      }
    }
  }

  // the four waves' results, one tile of queries after the other
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float sum = l[t] + __shfl_xor(l[t], 16);
    sum += __shfl_xor(sum, 32);
    if (lg == 0) {
      s_m[wave][ln] = m[t];
      s_l[wave][ln] = sum;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 8; i += 4)
        *reinterpret_cast<f32x4*>(&s_out[wave][ln][(lg * 4 + e) * 8 + i]) =
            f32x4{acc[t][i][e], acc[t][i + 1][e], acc[t][i + 2][e], acc[t][i + 3][e]};
    __syncthreads();
    const int n = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8, q = q0 + t * 16 + n;
    if (q < nq) {
      float top = s_m[0][n];
#pragma unroll
      for (int w = 1; w < 4; ++w) top = fmaxf(top, s_m[w][n]);
      const float from = top == -INFINITY ? 0.f : top;
      float total = 0.f, o[8] = {};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = s_m[w][n] == top ? 1.f : __builtin_amdgcn_exp2f(s_m[w][n] - from);
        total += s_l[w][n] * f;
        if (s_l[w][n] != 0.f)
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += s_out[w][n][d + e] * f;
      }
      const int i = q / rep, h = gr.g * rep + q - i * rep;
      const int64_t row = (int64_t)gr.b * r.per_request + i;
      if (p.splits == 1) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (bf16)(o[e] * inv);
        *reinterpret_cast<bf16x8*>((bf16*)r.out + row * r.out_ld + h * 128 + d) = v;
        if (r.lse && d == 0) r.lse[row * r.heads + h] = (from + __builtin_amdgcn_logf(total)) * kLn2;
      } else {
        const int64_t at = ((int64_t)gr.split * c.batch * r.per_request + row) * r.heads + h;
        *reinterpret_cast<f32x4*>(p.part + at * 128 + d) = f32x4{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<f32x4*>(p.part + at * 128 + d + 4) = f32x4{o[4], o[5], o[6], o[7]};
        if (d == 0) p.stats[at] = make_float2(top, total);
      }
    }
    __syncthreads();
  }
}

// fp32: 16 lanes share a key (elements lane % 16 + 16 i), a wave four keys at a
// time; every 16 lanes keep a running softmax of their own for the tile's four
// queries.
constexpr int kQueriesF32 = 4;
__global__ __launch_bounds__(256) void paged_attention_f32_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  constexpr int Q = kQueriesF32;
  __shared__ float s_out[16][128];
  __shared__ float s_m[16], s_l[16];
  Group gr;
  if (!group_of(c, p, gr)) return;
  const int ln = threadIdx.x & 15, str = threadIdx.x >> 4;  // 16 streams of keys
  const int rep = r.heads / c.kv_heads, nq = r.per_request * rep, q0 = gr.tile * Q, d = c.head_dim;
  int klen[Q], longest = 0;
  float q[Q][8], m[Q], l[Q], acc[Q][8];
  const float scale = kLog2e / sqrtf((float)d);
#pragma unroll
  for (int t = 0; t < Q; ++t) {
    const bool real = q0 + t < nq;
    const int i = real ? (q0 + t) / rep : 0;
    const int64_t row = (int64_t)gr.b * r.per_request + i;
    klen[t] = real ? capped_len(c, r.key_len[row]) : 0;
    longest = max(longest, klen[t]);
    const float* src = (const float*)r.q + row * r.q_ld + (int64_t)(gr.g * rep + (real ? q0 + t - i * rep : 0)) * d;
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      q[t][e] = ln + 16 * e < d ? src[ln + 16 * e] * scale : 0.f;
      acc[t][e] = 0.f;
    }
  }
  int begin, end;
  share_of(longest, p.splits, gr.split, begin, end);
  const int32_t* table = c.tables + (int64_t)gr.b * c.table_ld;
  for (int k = begin + str; k < end; k += 16) {
    const int slot = slot_of(c, table, k);
    const int64_t off = (int64_t)max(slot, 0) * c.ld + gr.g * d;
    float kv[8], vv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = slot >= 0 && ln + 16 * e < d;
      kv[e] = in ? ((const float*)c.k)[off + ln + 16 * e] : 0.f;
      vv[e] = in ? ((const float*)c.v)[off + ln + 16 * e] : 0.f;
    }
#pragma unroll
    for (int t = 0; t < Q; ++t) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s += q[t][e] * kv[e];
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) s += __shfl_xor(s, o);
      if (k >= klen[t] || s == -INFINITY) continue;  // uniform over the 16 lanes
      const float top = fmaxf(m[t], s);
      const float f = m[t] == top ? 1.f : __builtin_amdgcn_exp2f(m[t] - top);
      const float w = __builtin_amdgcn_exp2f(s - top);
      l[t] = l[t] * f + w;
      m[t] = top;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[t][e] = acc[t][e] * f + w * vv[e];
    }
  }
#pragma unroll
  for (int t = 0; t < Q; ++t) {
    if (ln == 0) {
      s_m[str] = m[t];
      s_l[str] = l[t];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) s_out[str][ln + 16 * e] = acc[t][e];
    __syncthreads();
    if (q0 + t < nq && (int)threadIdx.x < d) {
      float top = s_m[0];
      for (int w = 1; w < 16; ++w) top = fmaxf(top, s_m[w]);
      const float from = top == -INFINITY ? 0.f : top;
      float total = 0.f, o = 0.f;
      for (int w = 0; w < 16; ++w) {
        const float f = s_m[w] == top ? 1.f : __builtin_amdgcn_exp2f(s_m[w] - from);
        total += s_l[w] * f;
        if (s_l[w] != 0.f) o += s_out[w][threadIdx.x] * f;
      }
      const int i = (q0 + t) / rep, h = gr.g * rep + q0 + t - i * rep;
      const int64_t row = (int64_t)gr.b * r.per_request + i;
      if (p.splits == 1) {
        ((float*)r.out)[row * r.out_ld + (int64_t)h * d + threadIdx.x] = total == 0.f ? 0.f : o / total;
        if (r.lse && threadIdx.x == 0) r.lse[row * r.heads + h] = (from + __builtin_amdgcn_logf(total)) * kLn2;
      } else {
        const int64_t at = ((int64_t)gr.split * c.batch * r.per_request + row) * r.heads + h;
        p.part[at * d + threadIdx.x] = o;
        if (threadIdx.x == 0) p.stats[at] = make_float2(top, total);
      }
    }
    __syncthreads();
  }
}

// Joins the splits of a (row, head) in their order; a split without keys has a
// sum of 0 and is not read.  One wave, lane l elements 2 l and 2 l + 1.
template <typename T>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  const int64_t pairs = (int64_t)c.batch * r.per_request * r.heads;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= pairs) return;
  const int lane = threadIdx.x & 63, d = c.head_dim;
  float top = -INFINITY;
  for (int s = lane; s < p.splits; s += 64) top = fmaxf(top, p.stats[s * pairs + at].x);
  top = wave_max(top);
  const float from = top == -INFINITY ? 0.f : top;
  float total = 0.f, o[2] = {0.f, 0.f};
  for (int s = 0; s < p.splits; ++s) {
    const float2 st = p.stats[s * pairs + at];
    if (st.y == 0.f) continue;
    const float f = st.x == top ? 1.f : __builtin_amdgcn_exp2f(st.x - from);
    total += st.y * f;
    if (2 * lane < d) {
      const float2 v = *reinterpret_cast<const float2*>(p.part + (s * pairs + at) * d + 2 * lane);
      o[0] += v.x * f;
      o[1] += v.y * f;
    }
  }
  const int64_t row = at / r.heads, h = at - row * r.heads;
  if (2 * lane < d) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* dst = (T*)r.out + row * r.out_ld + h * d + 2 * lane;
    dst[0] = from_f32<T>(o[0] * inv);
    dst[1] = from_f32<T>(o[1] * inv);
  }
  if (r.lse && lane == 0) r.lse[at] = (from + __builtin_amdgcn_logf(total)) * kLn2;
}

int tile_queries(int queries, bool f32) { return f32 ? kQueriesF32 : queries <= 16 ? 16 : queries <= 32 ? 32 : 64; }

}  // namespace

hipError_t launch_paged_append(acache_dtype dt, const PagedCache& c, const AppendRows& r, float rope_base, hipStream_t s) {
  const double l2b = log2((double)rope_base);
  const int half = c.head_dim / 2, heads = (r.q ? r.heads : 0) + 2 * c.kv_heads;
  // a few rows: one to a workgroup, its items spread over several
  const int rows = r.n >= 2048 ? 4 : 1;
  auto go = [&](auto kernel, int v) {
    const int items = heads * (half / v);
    const int parts = rows > 1 ? 1 : std::min(64, (items + 255) / 256);
    hipLaunchKernelGGL(kernel, dim3((r.n + rows - 1) / rows, parts), dim3(256), (size_t)rows * half * sizeof(float2), s, c,
                       r, rows, l2b);
  };
  if (dt == ACACHE_BF16) go(paged_append_kernel<bf16, 8>, 8);
  else if (r.vec) go(paged_append_kernel<float, 4>, 4);
  else go(paged_append_kernel<float, 1>, 1);
  return hipGetLastError();
}

PagedPlan plan_paged_attention(acache_dtype dt, const PagedCache& c, int per_request, int heads, int64_t max_len,
                               size_t ws_bytes) {
  PagedPlan p = {};
  const int queries = per_request * (heads / c.kv_heads);
  p.tile = tile_queries(queries, dt == ACACHE_F32);
  p.tiles = (queries + p.tile - 1) / p.tile;
  const int64_t groups = (int64_t)c.batch * c.kv_heads * p.tiles;
  const int64_t pairs = (int64_t)c.batch * per_request * heads;
  // two workgroups for every CU, none with less than 128 keys
  int64_t splits = std::min<int64_t>((512 + groups - 1) / groups, (max_len + 127) / 128);
  const size_t each = (size_t)pairs * (c.head_dim + 2) * sizeof(float);
  splits = std::min<int64_t>(splits, (int64_t)(ws_bytes / std::max<size_t>(each, 1)));
  p.splits = (int)std::max<int64_t>(splits, 1);
  p.ws_bytes = p.splits > 1 ? p.splits * each : 0;
  return p;
}

hipError_t launch_paged_attention(acache_dtype dt, const PagedCache& c, const PagedQueries& r, const PagedPlan& plan,
                                  void* ws, hipStream_t s) {
  PagedPlan p = plan;
  const int64_t pairs = (int64_t)c.batch * r.per_request * r.heads;
  p.part = (float*)ws;
  p.stats = (float2*)(p.part + pairs * p.splits * c.head_dim);
  const int64_t keys = (int64_t)c.batch * c.kv_heads * p.splits;
  const dim3 grid((unsigned)((keys + 7) / 8 * 8 * p.tiles));
  if (dt == ACACHE_F32) hipLaunchKernelGGL(paged_attention_f32_kernel, grid, dim3(256), 0, s, c, r, p);
  else if (p.tile == 16) hipLaunchKernelGGL(paged_attention_kernel<1>, grid, dim3(256), 0, s, c, r, p);
  else if (p.tile == 32) hipLaunchKernelGGL(paged_attention_kernel<2>, grid, dim3(256), 0, s, c, r, p);
  else hipLaunchKernelGGL(paged_attention_kernel<4>, grid, dim3(256), 0, s, c, r, p);
  if (p.splits > 1) {
    const dim3 merge((unsigned)((pairs + 3) / 4));
    if (dt == ACACHE_F32) hipLaunchKernelGGL(paged_merge_kernel<float>, merge, dim3(256), 0, s, c, r, p);
    else hipLaunchKernelGGL(paged_merge_kernel<bf16>, merge, dim3(256), 0, s, c, r, p);
  }
  return hipGetLastError();
}

}  // namespace acache
