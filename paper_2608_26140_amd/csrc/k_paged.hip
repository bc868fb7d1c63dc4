// A cache in blocks with a table of block ids for each request: rotating and
// storing new rows, and attention of a step's rows over a request's positions.
//
// Position p of request b is slot tables[b][p / block] * block + p % block.  A
// position past the table, or whose entry names no block of the pools, has no
// slot: nothing is stored there, and it reads as a key and a value of zeros.
#include <algorithm>
#include <type_traits>

#include "device.h"
#include "internal.h"

namespace acache {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;

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
// one head: two runs of V elements, in and out.  A workgroup takes the items
// [256 blockIdx.y, + 256 gridDim.y, ..) of a row, whose angles it evaluates once
// (fp64, rotary_sincos) into LDS.  Bound by memory: each element is read and
// written once (8192 rows of 32 + 64 heads of 128 bf16, 403 MB: 77 us, 5.2 TB/s).
template <typename T, int V>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedCache c, AppendRows r, double log2_base) {
  extern __shared__ float2 turn[];  // [half]: cos, sin
  const int half = c.head_dim >> 1, per_head = half / V;
  const int heads = (r.q ? r.heads : 0) + 2 * c.kv_heads;
  const int items = heads * per_head;
  const int m = blockIdx.x, b = m / r.per_request, pos = r.pos[m];
  for (int i = threadIdx.x; i < half; i += 256) {
    float sn = 0.f, cs = 0.f;
    rotary_sincos((double)pos * exp2(-(2.0 * i / c.head_dim) * log2_base), &sn, &cs);
    turn[i] = make_float2(cs, sn);
  }
  __syncthreads();
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
        const float2 a = pos < 0 ? make_float2(0.f, 0.f) : turn[i + j];
        const float x = to_f32(lo.e[j]), y = to_f32(hi.e[j]);
        lo.e[j] = from_f32<T>(pos < 0 ? 0.f : x * a.x - y * a.y);
        hi.e[j] = from_f32<T>(pos < 0 ? 0.f : y * a.x + x * a.y);
      }
    }
    __builtin_memcpy(dst + i, &lo, sizeof(lo));
    __builtin_memcpy(dst + i + half, &hi, sizeof(hi));
  }
}

// ---------------------------------------------------------------- attention
constexpr int kMaxSplits = 256;

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

// The largest of a value in the four lanes lane % 16, + 16, + 32, + 48.
__device__ __forceinline__ float most_of_four(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Attention of 16 QT queries of a KV head over a share of the keys.  Four
// waves take 32 keys each at a time and keep their own running maximum, sum
// and output; they meet at the end.  A wave's rows of K and V are copied to LDS
// of its own a step ahead, 16-byte pieces of a row by adjacent lanes (a fragment's
// pieces straight from memory, 16 rows an instruction, keep the address unit busy
// for longer than the memory takes: one row of 1537 keys 18.5 us, 12.6 this way).
//  - S^T = K Q^T on MFMA 16x16x32: a lane's K fragment is 16 consecutive bytes
//    of a key's row; the result leaves a lane four keys (4 (lane / 16) + j) of two
//    16-key tiles for query lane % 16, whose maxima need two swaps between lanes;
//  - O^T = V^T P^T: those eight keys, in that order, are the lane's B fragment
//    (the order of the contraction is free), and for the A fragment a lane
//    reads 16 bytes of each of the same eight keys' rows, elements 8 (lane %
//    16) and on, and turns the 8 x 8 block in registers: row m of product i is
//    element 8 m + i.
// 16 KB are copied a step and wave; two workgroups share a CU, and their eight
// waves keep 128 KB in flight, several times what the memory's latency asks for
// at a CU's share of its rate.  The block ids of the next step's keys are on
// their way meanwhile.  Bound by memory up to some 32 queries of a KV head: a row
// each of 32 requests over 4352 keys, 32 heads, 1929 MB: 337 us, 5.7 TB/s; 32 rows
// of 8 requests over 2432 keys, 323 MB: 61 us, 5.3 TB/s.
// A weight is rounded to bf16 for its product with V (2^-8 relative at most); its sum
// is of the unrounded ones.  The maximum is kept exactly, so that the largest
// weight is 1, which rounding leaves as it is: raising it only in steps of 2^8
// saves 6% with 224 queries of a KV head, and takes the error against 64 bits
// from 0.0019 to 0.0026.
// Every lane finds the slot of one key and the others get it from there.  RUNS:
// blocks are of whole runs of 16 slots, so that the 16 keys of a tile lie one
// behind the other: their rows are a scalar base and per-lane offsets that do not
// change (2 x 16 rows of 28 heads on 4 over 8192 keys 20.9 us, 22.1 without; with
// one tile of queries, 32 requests or 1 over 1537 to 30011 keys, no difference).
template <int QT, bool RUNS>
__global__ __launch_bounds__(256, 2) void paged_attention_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  constexpr int LDO = 132;  // padded rows of the exchange
  struct Mine {             // a wave's: the rows on their way, then its results
    union {
      char rows[2][8192];
      float out[16 * QT][LDO];
    };
  };
  __shared__ __attribute__((aligned(1024))) Mine s_mine[4];
  __shared__ float s_m[4][16 * QT], s_l[4][16 * QT];
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

  // m: of the logits as they come from the product; weights 2^(scale (s - m))
  float m[QT], l[QT];
  f32x4 acc[QT][8];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Past the end the last key's block stands in: what is read there is masked.
  // RUNS: the blocks of the step's two tiles and where in them the tiles begin;
  // otherwise the block of key k0 + lane % 32.
  const int k_first = begin + wave * 32;
  auto last_at = [&](int k) { return min(k, end - 1); };
  auto block_at = [&](int k) { return table[(uint32_t)last_at(k) / (uint32_t)c.block]; };
  const int mine = RUNS ? 0 : lane & 31;
  int ahead[2] = {0, 0};
  if (k_first < end) {
    ahead[0] = block_at(k_first + mine);
    if (RUNS) ahead[1] = block_at(k_first + 16);
  }
  int slot[2], slot_next[2];  // of the tiles' first keys, or [0] of key k0 + mine
  auto slots_at = [&](int k0, int (&to)[2]) {  // takes the ids asked for, asks for the next ones
    auto slot_in = [&](int id, int k) {
      const int at = (int)((uint32_t)last_at(k) % (uint32_t)c.block);
      return id < 0 || id >= c.n_blocks ? -1 : id * c.block + (RUNS ? at & ~15 : at);
    };
    to[0] = slot_in(ahead[0], k0 + mine);
    to[1] = RUNS ? slot_in(ahead[1], k0 + 16) : 0;
    if (RUNS) {
      to[0] = __builtin_amdgcn_readfirstlane(to[0]);
      to[1] = __builtin_amdgcn_readfirstlane(to[1]);
    }
    ahead[0] = block_at(k0 + 128 + mine);
    if (RUNS) ahead[1] = block_at(k0 + 144);
  };
  // 16 copies of four whole rows each, in 16-byte pieces; K's pieces are laid
  // out so that the 16 keys of a fragment read distinct banks
  const uint32_t ld = (uint32_t)c.ld * 2u;  // bytes
  uint32_t k_off[4], v_off[4];              // in a tile
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    k_off[i] = (RUNS ? (i * 4 + lg) * ld : 0) + (ln ^ (i * 4 + lg)) * 16;
    v_off[i] = (RUNS ? (i * 4 + lg) * ld : 0) + ln * 16;
  }
  auto copy_rows = [&](const int (&from)[2]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int first = RUNS ? from[i >> 2] : __shfl(from[0], i * 4 + lg);
      const uint64_t at = (uint64_t)(uint32_t)max(first, 0) * ld;
      dma16((const char*)kp + at + k_off[i & 3], s_mine[wave].rows[0] + i * 1024);
      dma16((const char*)vp + at + v_off[i & 3], s_mine[wave].rows[1] + i * 1024);
    }
  };
  if (k_first < end) {
    slots_at(k_first, slot_next);
    copy_rows(slot_next);
  }
  for (int k0 = k_first; k0 < end; k0 += 128) {
    slot[0] = slot_next[0];
    slot[1] = slot_next[1];
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    u32x4 kr[2][4], vr[8];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        kr[t][k] = *reinterpret_cast<const u32x4*>(s_mine[wave].rows[0] + (t * 16 + ln) * 256 + ((k * 4 + lg) ^ ln) * 16);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      vr[e] = *reinterpret_cast<const u32x4*>(s_mine[wave].rows[1] + ((e & 4) * 4 + lg * 4 + (e & 3)) * 256 + ln * 16);
    wait_lgkmcnt<0>();  // the rows are read before the next ones come
    asm volatile("" ::: "memory");
    if (k0 + 128 < end) {
      slots_at(k0 + 128, slot_next);
      copy_rows(slot_next);
    }
    if (RUNS ? (slot[0] | slot[1]) < 0 : __ballot(slot[0] < 0) != 0) {  // keys without a slot are zeros
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if ((RUNS ? slot[t] : __shfl(slot[0], t * 16 + ln)) < 0)
#pragma unroll
          for (int k = 0; k < 4; ++k) kr[t][k] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((RUNS ? slot[e >> 2] : __shfl(slot[0], (e & 4) * 4 + lg * 4 + (e & 3))) < 0) vr[e] = u32x4{0, 0, 0, 0};
    }
    // An infinity or NaN of V at a key that some query does not attend to must
    // not reach it through a weight of 0: such elements are left out of the
    // product and added for the queries that do attend.
    const bool partly = k0 + 32 > shortest;
    bool odd = false;
    if (partly) {
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
            uint32_t y = vr[e][w];
            if ((y & 0x7F80u) == 0x7F80u) y &= 0xFFFF0000u;
            if ((y & 0x7F800000u) == 0x7F800000u) y &= 0xFFFFu;
            vr[e][w] = y;
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
    // the tiles of queries side by side, so that one's waits are the other's work
    f32x4 s[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) s[t][h] = mfma16(__builtin_bit_cast(bf16x8, kr[h][k]), qf[t][k], s[t][h]);
    if (partly)
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[t][h][j] = k0 + h * 16 + lg * 4 + j < klen[t] ? s[t][h][j] : -INFINITY;
    float top[QT];
    bool rises = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      top[t] = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) top[t] = fmaxf(top[t], s[t][h][j]);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      top[t] = most_of_four(top[t]);
      rises |= top[t] > m[t];
    }
    if (__ballot(rises))
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const bool up = top[t] > m[t];
        const float f = up ? __builtin_amdgcn_exp2f((m[t] - top[t]) * scale) : 1.f;
        l[t] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[t][i] *= f;
        m[t] = up ? top[t] : m[t];
      }
    bf16x8 pf[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float from = m[t] == -INFINITY ? 0.f : m[t] * scale;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float w = __builtin_amdgcn_exp2f(fmaf(s[t][h][j], scale, -from));
          s[t][h][j] = w;
          l[t] += w;
          pf[t][h * 4 + j] = (bf16)w;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int t = 0; t < QT; ++t) acc[t][i] = mfma16(va[i], pf[t], acc[t][i]);
    if (odd) {
#pragma unroll 1
      for (int key = 0; key < 32; ++key) {
        const int run = slot[key >> 4 & (RUNS ? 1 : 0)];
        const int64_t at = RUNS ? (run < 0 ? -1 : run + (key & 15)) : __shfl(slot[0], key);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          float w = 0.f;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key >> 4 == h && (key & 3) == j) w = s[t][h][j];
          w = (float)(bf16)__shfl(w, (key & 12) * 4 + ln);
          const bool seen = k0 + key < klen[t] && at >= 0;
          const bf16* src = vp + (seen ? at * c.ld : 0) + lg * 32;
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

  // the four waves' results
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float sum = l[t] + __shfl_xor(l[t], 16);
    sum += __shfl_xor(sum, 32);
    if (lg == 0) {
      s_m[wave][t * 16 + ln] = m[t] * scale;
      s_l[wave][t * 16 + ln] = sum;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 8; i += 4)
        *reinterpret_cast<f32x4*>(&s_mine[wave].out[t * 16 + ln][(lg * 4 + e) * 8 + i]) =
            f32x4{acc[t][i][e], acc[t][i + 1][e], acc[t][i + 2][e], acc[t][i + 3][e]};
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int n = t * 16 + (threadIdx.x >> 4), d = (threadIdx.x & 15) * 8, q = q0 + n;
    if (q >= nq) continue;
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
        for (int e = 0; e < 8; ++e) o[e] += s_mine[w].out[n][d + e] * f;
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
}

// Attention of 128 queries of a KV head, 32 to a wave, where there are that
// many: tiles of 64 keys pass through LDS once for all four waves (two tiles, so
// that one is copied while the other is read; a barrier a tile), and no two
// waves' results have to be joined.  Blocks are of whole runs of 16 slots; a
// wave copies one run of the tile, its pieces laid out so that the products'
// fragments are read from distinct banks.
//  - S^T = K Q^T on MFMA 32x32x16: a lane has query lane % 32 and, rows of K
//    taken in the order of key_row, keys 16 (r / 8) + 8 (lane / 32) + r % 8 of
//    each 32 in register r: what the second product wants of P;
//  - O^T = V^T P^T, V's fragments by transposing reads.
// Bound by its work: per tile and wave 32 products of 32 cycles, 32 exponentials
// of 16 and some 200 other vector instructions, about half of what 32 queries
// with keys of their own take (paged_attention_kernel): 4 x 256 rows of 28 heads
// over 4096 keys 88 us, 0.68 PFLOP/s.
typedef __attribute__((__vector_size__(4 * sizeof(int16_t)))) int16_t i16x4;
__device__ __forceinline__ i16x4 read_turned(const char* lds) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)lds);
}
__device__ __forceinline__ int key_row(int m) { return (m >> 4) * 16 + ((m >> 2) & 1) * 8 + ((m >> 3) & 1) * 4 + (m & 3); }
__device__ __forceinline__ int v_swizzle(int row) { return ((row & 3) << 2) ^ (row & 1); }

constexpr int kWideQueries = 128;
__global__ __launch_bounds__(256, 2) void paged_attention_wide_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  constexpr int TILE = 64, ROW = 256, HALF = TILE * ROW;
  __shared__ __attribute__((aligned(1024))) char s_tile[2][2 * HALF];  // K, V
  __shared__ int s_len[4];
  Group gr;
  if (!group_of(c, p, gr)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qn = lane & 31, hl = lane >> 5, ln = lane & 15, lg = lane >> 4;
  const int rep = r.heads / c.kv_heads, nq = r.per_request * rep;
  const int q = gr.tile * kWideQueries + wave * 32 + qn;
  const bool real = q < nq, live = gr.tile * kWideQueries + wave * 32 < nq;
  const int qi = real ? q / rep : 0, h = gr.g * rep + (real ? q - qi * rep : 0);
  const int64_t row = (int64_t)gr.b * r.per_request + qi;
  const int klen = real ? capped_len(c, r.key_len[row]) : 0;
  bf16x8 qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s)
    qf[s] = *reinterpret_cast<const bf16x8*>((const bf16*)r.q + row * r.q_ld + h * 128 + s * 16 + hl * 8);
  int longest = klen, shortest = real ? klen : 0x7FFFFFFF;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    longest = max(longest, __shfl_xor(longest, o));
    shortest = min(shortest, __shfl_xor(shortest, o));
  }
  if (lane == 0) s_len[wave] = longest;
  __syncthreads();
  longest = max(max(s_len[0], s_len[1]), max(s_len[2], s_len[3]));
  longest = __builtin_amdgcn_readfirstlane(longest);
  shortest = __builtin_amdgcn_readfirstlane(shortest);

  int begin, end;
  share_of(longest, p.splits, gr.split, begin, end);
  const int32_t* table = c.tables + (int64_t)gr.b * c.table_ld;
  const float scale = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)

  // copies: run `wave` of a tile, four rows an instruction
  const uint32_t ld = (uint32_t)c.ld * 2u;
  const char* kp = (const char*)c.k + gr.g * 256;
  const char* vp = (const char*)c.v + gr.g * 256;
  // (row i * 4 + lg of the run: the swizzles of its pieces are ln ^ lg ^ 4 i, and
  // the same in every i)
  const uint32_t k_piece = ln ^ lg, row_off = lg * ld, v_off = row_off + (ln ^ v_swizzle(lg)) * 16;
  auto last_at = [&](int k) { return min(k, end - 1); };
  auto block_at = [&](int k) { return table[(uint32_t)last_at(k) / (uint32_t)c.block]; };
  int ahead = begin < end ? block_at(begin + wave * 16) : 0;
  auto copy_tile = [&](int k0, int stage) {
    const int at = (int)((uint32_t)last_at(k0 + wave * 16) % (uint32_t)c.block) & ~15;
    const int id = __builtin_amdgcn_readfirstlane(ahead);
    ahead = block_at(k0 + TILE + wave * 16);
    char* to = s_tile[stage] + wave * 16 * ROW;
    if (id >= 0 && id < c.n_blocks) {
      const uint64_t from = (uint64_t)(uint32_t)(id * c.block + at) * ld;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dma16_global_asm(kp + from + (uint64_t)(4 * i) * ld + (row_off + ((k_piece ^ (4 * i)) << 4)), to + i * 1024);
        dma16_global_asm(vp + from + (uint64_t)(4 * i) * ld + v_off, to + HALF + i * 1024);
      }
    } else {  // keys without a slot are zeros
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x4*>(to + i * 1024 + lane * 16) = *reinterpret_cast<u32x4*>(to + HALF + i * 1024 + lane * 16) =
            u32x4{0, 0, 0, 0};
    }
  };

  f32x16 acc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int k_row = key_row(qn), v_row = 8 * (lg >> 1) + (ln >> 2), v_col = 2 * (lg & 1) + ((ln & 3) >> 1);
  if (begin < end) copy_tile(begin, 0);
  int stage = 0;
  auto take = [&](auto masked, int k0) {
    wait_vmcnt<0>();
    wait_lgkmcnt<0>();
    bare_barrier();  // the tile is there, and nobody reads the other one
    if (k0 + TILE < end) copy_tile(k0 + TILE, stage ^ 1);
    const char* kt = s_tile[stage];
    const char* vt = kt + HALF;
    stage ^= 1;
    if (!live) return;
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
    for (int st = 0; st < 8; ++st)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + (kb * 32 + k_row) * ROW + (((2 * st + hl) ^ (k_row & 15)) << 4));
        s[kb] = mfma32x32x16(kf, qf[st], s[kb]);
      }
    if constexpr (masked.value)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[kb][i] = k0 + kb * 32 + 16 * (i >> 3) + 8 * hl + (i & 7) < klen ? s[kb][i] : -INFINITY;
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    if (__ballot(top > m)) {
      const bool up = top > m;
      const float f = up ? __builtin_amdgcn_exp2f((m - top) * scale) : 1.f;
      l *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= f;
      m = up ? top : m;
    }
    const float from = m == -INFINITY ? 0.f : m * scale;
    bf16x8 pf[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[kb][i], scale, -from));
        s[kb][i] = w;
        l += w;
        pf[kb * 2 + (i >> 3)][i & 7] = (bf16)w;
      }
    u16x2 least = {1, 1};  // 0: an infinity or NaN of V where some query does not attend (see above)
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const char* at = vt + (g * 16 + v_row) * ROW + (((4 * d + v_col) ^ v_swizzle(v_row)) << 4) + (ln & 1) * 8;
          const i16x4 lo = read_turned(at), hi = read_turned(at + 4 * ROW);
          u32x4 vf = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          if constexpr (masked.value)
#pragma unroll
            for (int w = 0; w < 4; ++w) {  // both halves at a time: 0 where the exponent is all ones
              const uint32_t word = vf[w];
              const u16x2 y = __builtin_bit_cast(u16x2, word);
              const u16x2 rest = __builtin_elementwise_min((y & (u16x2){0x7F80, 0x7F80}) ^ (u16x2){0x7F80, 0x7F80}, (u16x2){1, 1});
              least = __builtin_elementwise_min(least, rest);
              vf[w] = __builtin_bit_cast(uint32_t, y & ((u16x2){0, 0} - rest));
            }
          acc[d] = mfma32x32x16(__builtin_bit_cast(bf16x8, vf), pf[g], acc[d]);
        }
    if constexpr (masked.value)
      if (__ballot((least[0] & least[1]) == 0)) {
#pragma unroll 1
      for (int key = 0; key < TILE; ++key) {
        float w = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (key >> 5 == kb && ((key >> 4) & 1) * 8 + (key & 7) == i) w = s[kb][i];
        w = (float)(bf16)__shfl(w, qn + ((key >> 3) & 1) * 32);
        const bool seen = k0 + key < klen;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int e = d * 32 + 8 * (i >> 2) + 4 * hl + (i & 3);
            const bf16 x = *reinterpret_cast<const bf16*>(vt + key * ROW + (((e >> 3) ^ v_swizzle(key)) << 4) + (e & 7) * 2);
            const float v = to_f32(x);
            if (seen && !(fabsf(v) < INFINITY)) acc[d][i] += w * v;
          }
      }
    }
  };
  // tiles that all of the wave's queries attend to whole, then the others
  int k0 = begin;
  for (; k0 < end && k0 + TILE <= shortest; k0 += TILE) take(std::false_type{}, k0);
  for (; k0 < end; k0 += TILE) take(std::true_type{}, k0);

  if (!real) return;
  const float total = l + __shfl_xor(l, 32);
  if (p.splits == 1) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    bf16* dst = (bf16*)r.out + row * r.out_ld + h * 128 + 4 * hl;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16)(acc[d][i + e] * inv);
        *reinterpret_cast<bf16x4*>(dst + d * 32 + 2 * i) = v;
      }
    if (r.lse && hl == 0) r.lse[row * r.heads + h] = ((m == -INFINITY ? 0.f : m * scale) + __builtin_amdgcn_logf(total)) * kLn2;
  } else {
    const int64_t at = ((int64_t)gr.split * c.batch * r.per_request + row) * r.heads + h;
    float* dst = p.part + at * 128 + 4 * hl;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(dst + d * 32 + 2 * i) = f32x4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
    if (hl == 0) p.stats[at] = make_float2(m * scale, total);
  }
}

// fp32: 16 lanes share a key (elements lane % 16 + 16 i), a wave four keys at a
// time, four such on their way; every 16 lanes keep a running softmax of their
// own for the tile's four queries, four keys of it at a time.  Bound by the
// latency of a step (block id, rows, sums over 16 lanes): 5 rows of 3 requests
// over 403 keys, 4 heads of 32 on 2: 11.9 us with the join, 17.4 with a softmax
// step for each key and a join of the 16 streams by one thread an element; 5 rows
// of each of 16 requests over 4096 keys, 8 heads of 128 on 4: 148 us, three times
// what the bytes take.  Measured there and no better: block ids asked for a step ahead (151),
// pairs of elements by one load (155).
constexpr int kQueriesF32 = 4;

// The sum over the 16 lanes of a row, in each of them (moves in registers: by
// half the row, a quarter, ...).
template <int ROR>
__device__ __forceinline__ float turned_row(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + ROR, 0xF, 0xF, false));
}
__device__ __forceinline__ float row_sum(float v) {
  v += turned_row<8>(v);
  v += turned_row<4>(v);
  v += turned_row<2>(v);
  v += turned_row<1>(v);
  return v;
}

template <int N>  // elements of a head that a lane has, head_dim <= 16 N
__global__ __launch_bounds__(256) void paged_attention_f32_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  constexpr int Q = kQueriesF32, U = 4;
  static_assert(Q == 4, "a wave joins a query");
  __shared__ float s_out[16][Q][16 * N];
  __shared__ float s_m[Q][16], s_l[Q][16];
  Group gr;
  if (!group_of(c, p, gr)) return;
  const int ln = threadIdx.x & 15, str = threadIdx.x >> 4;  // 16 streams of keys
  const int rep = r.heads / c.kv_heads, nq = r.per_request * rep, q0 = gr.tile * Q, d = c.head_dim;
  int klen[Q], longest = 0, shortest = 0x7FFFFFFF;
  float q[Q][N], m[Q], l[Q], acc[Q][N];
  const float scale = kLog2e / sqrtf((float)d);
#pragma unroll
  for (int t = 0; t < Q; ++t) {
    const bool real = q0 + t < nq;
    const int i = real ? (q0 + t) / rep : 0;
    const int64_t row = (int64_t)gr.b * r.per_request + i;
    klen[t] = real ? capped_len(c, r.key_len[row]) : 0;
    longest = max(longest, klen[t]);
    if (real) shortest = min(shortest, klen[t]);
    const float* src = (const float*)r.q + row * r.q_ld + (int64_t)(gr.g * rep + (real ? q0 + t - i * rep : 0)) * d;
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      q[t][e] = ln + 16 * e < d ? src[ln + 16 * e] * scale : 0.f;
      acc[t][e] = 0.f;
    }
  }
  int begin, end;
  share_of(longest, p.splits, gr.split, begin, end);
  const int32_t* table = c.tables + (int64_t)gr.b * c.table_ld;
  for (int k0 = begin; k0 < end; k0 += 16 * U) {
    int slot[U];
    float kv[U][N], vv[U][N], s[U][Q];
#pragma unroll
    for (int u = 0; u < U; ++u) slot[u] = k0 + 16 * u + str < end ? slot_of(c, table, k0 + 16 * u + str) : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t off = (int64_t)max(slot[u], 0) * c.ld + gr.g * d;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const bool in = slot[u] >= 0 && ln + 16 * e < d;
        kv[u][e] = in ? ((const float*)c.k)[off + ln + 16 * e] : 0.f;
        vv[u][e] = in ? ((const float*)c.v)[off + ln + 16 * e] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < Q; ++t) {
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) x += q[t][e] * kv[u][e];
        s[u][t] = row_sum(x);
      }
    const bool whole = k0 + 16 * U <= shortest;  // for every query
#pragma unroll
    for (int t = 0; t < Q; ++t) {
      float top = m[t];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!whole) s[u][t] = k0 + 16 * u + str < klen[t] ? s[u][t] : -INFINITY;
        top = fmaxf(top, s[u][t]);
      }
      const float f = m[t] == top ? 1.f : __builtin_amdgcn_exp2f(m[t] - top), from = top == -INFINITY ? 0.f : top;
      m[t] = top;
      l[t] *= f;
#pragma unroll
      for (int e = 0; e < N; ++e) acc[t][e] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = __builtin_amdgcn_exp2f(s[u][t] - from);
        l[t] += w;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[t][e] += w * (whole || s[u][t] != -INFINITY ? vv[u][e] : 0.f);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < Q; ++t) {
    if (ln == 0) {
      s_m[t][str] = m[t];
      s_l[t][str] = l[t];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) s_out[str][t][ln + 16 * e] = acc[t][e];
  }
  __syncthreads();
  // wave t joins the 16 streams of query t
  const int t = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (q0 + t >= nq) return;
  const float own = s_m[t][ln], own_l = s_l[t][ln];
  float top = own;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float from = top == -INFINITY ? 0.f : top;
  const float f = own_l == 0.f ? 0.f : own == top ? 1.f : __builtin_amdgcn_exp2f(own - from);
  const float total = row_sum(own_l * f);
  const int i = (q0 + t) / rep, h = gr.g * rep + q0 + t - i * rep;
  const int64_t row = (int64_t)gr.b * r.per_request + i;
  const int64_t at = ((int64_t)gr.split * c.batch * r.per_request + row) * r.heads + h;
  for (int e = lane; e < d; e += 64) {
    float o = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const float fw = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(f), w));
      if (fw != 0.f) o += s_out[w][t][e] * fw;
    }
    if (p.splits == 1) ((float*)r.out)[row * r.out_ld + (int64_t)h * d + e] = total == 0.f ? 0.f : o / total;
    else p.part[at * d + e] = o;
  }
  if (lane == 0) {
    if (p.splits > 1) p.stats[at] = make_float2(top, total);
    else if (r.lse) r.lse[row * r.heads + h] = (from + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

// Joins the splits of a (row, head), a split without keys (sum 0) is not read.
// WAVES waves take every WAVES-th split, eight at a time, lane l elements 2 l and
// 2 l + 1, and are added in their order.
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedCache c, PagedQueries r, PagedPlan p) {
  __shared__ float2 s_part[WAVES > 1 ? WAVES : 1][64];
  const int64_t pairs = (int64_t)c.batch * r.per_request * r.heads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = c.head_dim;
  const int64_t at = WAVES > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  if (at >= pairs) return;
  constexpr int NS = (kMaxSplits + 63) / 64;
  float2 st[NS];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    st[i] = make_float2(-INFINITY, 0.f);
    if (i * 64 < p.splits && i * 64 + lane < p.splits) st[i] = p.stats[(i * 64 + lane) * pairs + at];
    top = fmaxf(top, st[i].x);
  }
  top = wave_max(top);
  const float from = top == -INFINITY ? 0.f : top;
  float total = 0.f, f[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    f[i] = st[i].x == top ? 1.f : __builtin_amdgcn_exp2f(st[i].x - from);
    total += st[i].y * f[i];
    if (st[i].y == 0.f) f[i] = 0.f;
  }
  total = wave_sum(total);
  float2 o = make_float2(0.f, 0.f);
  const float* part = p.part + at * d + 2 * lane;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    if (i * 64 >= p.splits) break;
    const int n = min(64, p.splits - i * 64);
    for (int j0 = WAVES > 1 ? wave : 0; j0 < n; j0 += 8 * WAVES) {
      float2 v[8];
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int s = j0 + j * WAVES;
        w[j] = s < n ? __shfl(f[i], s) : 0.f;
        v[j] = make_float2(0.f, 0.f);
        if (w[j] != 0.f && 2 * lane < d) v[j] = *reinterpret_cast<const float2*>(part + (int64_t)(i * 64 + s) * pairs * d);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o.x += v[j].x * w[j];
        o.y += v[j].y * w[j];
      }
    }
  }
  if constexpr (WAVES > 1) {
    s_part[wave][lane] = o;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      o.x += s_part[w][lane].x;
      o.y += s_part[w][lane].y;
    }
  }
  const int64_t row = at / r.heads, h = at - row * r.heads;
  if (2 * lane < d) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* dst = (T*)r.out + row * r.out_ld + h * d + 2 * lane;
    dst[0] = from_f32<T>(o.x * inv);
    dst[1] = from_f32<T>(o.y * inv);
  }
  if (r.lse && lane == 0) r.lse[at] = (from + __builtin_amdgcn_logf(total)) * kLn2;
}

// Blocks are of whole runs of 16 slots, 16 rows of which lie within 2^31 bytes.
bool in_runs(const PagedCache& c) { return c.block % 16 == 0 && c.ld < 1 << 26; }

// Shares of the keys of all requests and KV heads, in whole rounds of the XCDs
// (group_of): each takes a workgroup for every query tile.
int64_t paged_groups(const PagedCache& c, int64_t splits) { return ((int64_t)c.batch * c.kv_heads * splits + 7) / 8 * 8; }

// Tiles of 16 for up to 16 queries: 7 of each of 4 KV heads of 8 requests over 8192
// keys 31.3 us, 33.7 with tiles of 32; 28 of each 47.9, 37.1.
// Tiles of 128 from 193 queries on, where both of a KV head's first two are more
// than half full: 4 x 32 rows of 28 heads on 4 (224 queries) over 5120 keys 27.4 us,
// 31.5 with tiles of 32; 4 x 64 rows 40.3, 52.2; 4 x 256 rows (1792) over 4096 keys
// 88, 113; but 160 queries of one KV head over 3000 keys 11.8, 11.1.
int tile_queries(int64_t queries, bool f32, bool runs) {
  if (f32) return kQueriesF32;
  if (runs && queries > 192) return kWideQueries;
  return queries <= 16 ? 16 : 32;
}

}  // namespace

hipError_t launch_paged_append(acache_dtype dt, const PagedCache& c, const AppendRows& r, float rope_base, hipStream_t s) {
  const double l2b = log2((double)rope_base);
  const int half = c.head_dim / 2, heads = (r.q ? r.heads : 0) + 2 * c.kv_heads;
  // Below 1024 rows a row's items are spread over workgroups, each with all of its
  // angles: 128 rows of 32 + 64 heads 3.4 us, 4.1 with one; from there on one takes
  // them all: 4096 rows 35.7, spread 39.7, 8192 of 28 + 8 heads 30.5, 40.
  auto go = [&](auto kernel, int v) {
    const int parts = r.n >= 1024 ? 1 : std::min(64, (heads * (half / v) + 255) / 256);
    hipLaunchKernelGGL(kernel, dim3(r.n, parts), dim3(256), (size_t)half * sizeof(float2), s, c, r, l2b);
  };
  if (dt == ACACHE_BF16) go(paged_append_kernel<bf16, 8>, 8);
  else if (r.vec) go(paged_append_kernel<float, 4>, 4);
  else go(paged_append_kernel<float, 1>, 1);
  return hipGetLastError();
}

PagedPlan plan_paged_attention(acache_dtype dt, const PagedCache& c, int per_request, int heads, int64_t max_len,
                               size_t ws_bytes) {
  PagedPlan p = {};
  const int64_t queries = (int64_t)per_request * (heads / c.kv_heads);
  p.tile = tile_queries(queries, dt == ACACHE_F32, in_runs(c));
  const int64_t tiles = (queries + p.tile - 1) / p.tile;
  const int64_t groups = (int64_t)c.batch * c.kv_heads * tiles;
  const int64_t pairs = (int64_t)c.batch * per_request * heads;
  const size_t each = (size_t)pairs * (c.head_dim + 2) * sizeof(float);
  // a launch has less than 2^24 workgroups of 256 threads
  constexpr int64_t kMost = 1 << 24;
  auto fits = [&](int64_t splits) { return paged_groups(c, splits) * tiles < kMost; };
  if (!fits(1)) return p;
  p.tiles = (int)tiles;
  const int64_t most = pairs >= kMost ? 1
                                      : std::min<int64_t>({(max_len + 127) / 128, kMaxSplits,
                                                           (int64_t)(ws_bytes / std::max<size_t>(each, 1))});
  // The split with the least estimated time, in us.  Workgroups run two a CU, in
  // rounds; one takes a step for every 128 keys.  A step is the longest of a
  // chain of dependent waits that grows with the load, the rate of the memory for
  // all that run (6 TB/s; tiles of the same keys read them once), and the work of
  // those that share a CU.  The join is a launch, and the partials' way.  One row
  // of 8 requests over 30011 keys, 4 KV heads: 321 us unsplit, 96 in 5 parts, 85
  // in 8, 84 in 16, 92 in 32; 4 x 32 rows of 28 heads over 5120 keys: 108, 2 parts
  // 64, 4 parts 39, 8 parts 28, 16 parts 34.
  const bool f32 = dt == ACACHE_F32;
  const double chain = f32 ? 2.0 : p.tile == kWideQueries ? 2.6 : p.tile == 32 ? 1.1 : 1.3;
  const double work = f32 ? 1.5 : p.tile == kWideQueries ? 2.8 : p.tile == 32 ? 1.05 : 0.6;
  int64_t splits = 1;
  double best = 1e30;
  for (int64_t s = 1; s <= std::max<int64_t>(most, 1) && fits(s); ++s) {
    const int64_t n = groups * s, running = std::min<int64_t>(n, 512);
    const double read = running * 256.0 * c.head_dim * (f32 ? 4 : 2) / 6e6 / p.tiles;
    const double step = std::max({chain + 0.35 * read, read, work * (double)((running + 255) / 256)});
    const double steps = (double)(((max_len + s - 1) / s + 127) / 128);
    const double us = 4.0 + (steps * step + 1.6) * (n > 512 ? n / 512.0 + 0.3 : 1.0) +
                      (s > 1 ? 4.0 + 0.05 * s + (double)s * pairs * c.head_dim / 1e6 : 0.0);
    if (us < best) {
      best = us;
      splits = s;
    }
  }
  p.splits = (int)splits;
  p.ws_bytes = p.splits > 1 ? p.splits * each : 0;
  return p;
}

hipError_t launch_paged_attention(acache_dtype dt, const PagedCache& c, const PagedQueries& r, const PagedPlan& plan,
                                  void* ws, hipStream_t s) {
  PagedPlan p = plan;
  const int64_t pairs = (int64_t)c.batch * r.per_request * r.heads;
  p.part = (float*)ws;
  p.stats = (float2*)(p.part + pairs * p.splits * c.head_dim);
  const dim3 grid((unsigned)(paged_groups(c, p.splits) * p.tiles));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, c, r, p); };
  if (dt == ACACHE_F32) {
    // 16 requests of 5 rows, 8 heads of 32 on 4, over 4096 keys: 53 us, 92 with the
    // elements of a head of 128; heads of 64: 79, 104
    if (c.head_dim <= 32) go(paged_attention_f32_kernel<2>);
    else if (c.head_dim <= 64) go(paged_attention_f32_kernel<4>);
    else go(paged_attention_f32_kernel<8>);
  } else {
    if (p.tile == kWideQueries) go(paged_attention_wide_kernel);
    else if (p.tile == 16) go(paged_attention_kernel<1, false>);
    else in_runs(c) ? go(paged_attention_kernel<2, true>) : go(paged_attention_kernel<2, false>);
  }
  if (p.splits > 1) {
    // one wave a pair with up to 8 splits (4 x 32 rows of 28 heads in 8: 27.5 us,
    // 33.4 with four waves), else four (one row of 32 heads in 13: 11.9, 12.7)
    const dim3 few((unsigned)((pairs + 3) / 4)), many((unsigned)pairs);
    if (dt == ACACHE_F32 && p.splits <= 8) hipLaunchKernelGGL((paged_merge_kernel<float, 1>), few, dim3(256), 0, s, c, r, p);
    else if (dt == ACACHE_F32) hipLaunchKernelGGL((paged_merge_kernel<float, 4>), many, dim3(256), 0, s, c, r, p);
    else if (p.splits <= 8) hipLaunchKernelGGL((paged_merge_kernel<bf16, 1>), few, dim3(256), 0, s, c, r, p);
    else hipLaunchKernelGGL((paged_merge_kernel<bf16, 4>), many, dim3(256), 0, s, c, r, p);
  }
  return hipGetLastError();
}

}  // namespace acache
