// Read-slot attention over the 8-bit KV cache (gfx950): softmax(q K^T) V with
// keys and values gathered through a slot map, K = code * 2^e of its block.
//
// What is read from memory is the codes; a workgroup turns each key and value
// into bf16 once for all its queries (code * 2^e is exact in bf16, and one
// instruction converts and scales two codes), and both products run on the
// bf16 MFMA with fp32 sums.  The 8-bit MFMA would take K as it lies in the
// cache, with each bf16 query split into two 8-bit numbers, in the same time,
// but it drops what lies 2^-13 and less below a product's largest term
// (measured: 64 terms over eight binades, errors up to 2^-13 of the largest
// term), which the logits and their log-sum-exp would show.
// Each lane owns one query (in-lane softmax statistics plus one exchange
// between the lane halves); a fixed key permutation inside each 16-key group
// makes the lane's weights line up as the second product's B operand, and V
// is read as V^T through transposing LDS reads.  Softmax runs in base 2 with a
// running maximum that moves only when exceeded by more than 2^8.  Logits,
// weights' sum and output are held in fp32; a weight is rounded to bf16 for
// the product with V, half a step of 2^-8 of it, as in the bf16 attention: the
// fp32 product has a sixteenth of the bf16 one's rate.  Against 64 bits the
// outputs are off by 0.0017 to 0.0022 (relative); by 0.0017 with fp32 weights,
// which is the rounding of the bf16 output.
//
// With grouped heads the query heads of a KV head are further queries of the
// same tile: a request's query v is row v mod rows of head g rep + v / rows.
// Two kernels share the work (launch_quant_attention): 256 queries a
// workgroup, or 32 with the keys dealt to its waves.
#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "quant.h"

namespace acache {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef short v4i16 __attribute__((__vector_size__(4 * sizeof(short))));

constexpr int kDh = 128;
constexpr int kTileK = 64;             // keys per tile
constexpr int kRowB = kDh * 2;                // a converted row
constexpr int kTileB = kTileK * kRowB;        // 16 KB: a converted tile
constexpr int kAuxB = kTileK * 4;             // a 32-bit value for each key of a tile
constexpr int kMaxSplits = 64;
// buffer offset of an absent key: past every pool the entry point admits, so
// its copies give zeros
constexpr uint32_t kAbsent = 0xF0000000u;

struct QAttnArgs {
  QuantPool p;
  const bf16* q;
  const int32_t* slots;
  bf16* out;
  float* lse;
  float* part_o;   // [splits][rows][H][128] unnormalised O (splits > 1)
  float* part_ml;  // [splits][rows][H][2] (running max in log2 units, sum)
  int H, rep, splits;
  Ragged rg;       // tile_start: this launch's query tiles of a KV head
  // this launch's queries of request b: v_lo[b] .. v_hi[b] - 1 of its rows * rep
  int v_lo[kMaxBatch], v_hi[kMaxBatch];
};

// key (within a 32-key block) that S^T row i holds
__device__ __forceinline__ int key_perm(int i) {
  const int r = i & 15;
  return (i & 16) | (8 * ((r >> 2) & 1) + (r & 3) + 4 * (r >> 3));
}
__device__ __forceinline__ v4i16 ds_read_tr16(const char* lds) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16*)lds);
}

// Q^T fragments of a lane's query: dimensions 16 s + 8 hl .. + 7.
__device__ __forceinline__ void load_query(const bf16* q, bool ok, int hl, bf16x8 (&f)[8]) {
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (ok) v = *reinterpret_cast<const u32x4*>(q + 16 * s + 8 * hl);
    f[s] = __builtin_bit_cast(bf16x8, v);
  }
}

// 16 codes times 2^e (scale's exponent) as 16 bf16
__device__ __forceinline__ void convert16(u32x4 w, float scale, u32x4 (&v)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i >> 1][2 * (i & 1)] =
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
    v[i >> 1][2 * (i & 1) + 1] =
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
  }
}

// The (KV head, request, query tile, key split) of a workgroup: an eighth of
// the grid on each XCD, KV heads outermost, `side` of them next to each other.
struct Unit {
  int g, b, tile, split;
};
__device__ __forceinline__ Unit unit_of(const Ragged& rg, int splits, int side) {
  const int n_tiles = rg.tile_start[rg.batch];
  const int nb = gridDim.x, i = blockIdx.x;
  const int q8 = nb >> 3, r8 = nb & 7, x = i & 7;
  const int t = x * q8 + min(x, r8) + (i >> 3);
  Unit u;
  const int group = t / (n_tiles * splits * side);
  int rem = t - group * (n_tiles * splits * side);
  u.g = group * side + rem % side;
  rem /= side;
  u.tile = rem / splits;
  u.split = rem - u.tile * splits;
  int lo = 0, hi = rg.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (rg.tile_start[mid] <= u.tile) lo = mid; else hi = mid - 1;
  }
  u.b = lo;
  u.tile -= rg.tile_start[lo];
  return u;
}

// Writes a lane's query: the output and its log-sum-exp, or a split's partial.
// O^T register r of block d holds dimension 32 d + 8 (r / 4) + 4 hl + r % 4.
__device__ __forceinline__ void write_query(const QAttnArgs& a, int64_t pair, int split, int hl, const f32x16 (&o)[4],
                                            float m, float l) {
  if (a.splits > 1) {
    const int64_t pairs = (int64_t)a.rg.cu_rows[a.rg.batch] * a.H;
    float* po = a.part_o + (split * pairs + pair) * kDh;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = {o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]};
        *reinterpret_cast<f32x4*>(po + d * 32 + 8 * q + 4 * hl) = v;
      }
    if (hl == 0) *reinterpret_cast<float2*>(a.part_ml + (split * pairs + pair) * 2) = float2{m, l};
    return;
  }
  if (a.lse && hl == 0) a.lse[pair] = (m + __log2f(l)) * kLn2;
  const float inv = 1.f / l;
  bf16* op = a.out + pair * kDh;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (bf16)(o[d][4 * q + j] * inv);
      *reinterpret_cast<bf16x4*>(op + d * 32 + 8 * q + 4 * hl) = w;
    }
}

// ============================================================================
// quant_attention_wide_kernel: 256 queries of one KV head and request a
// workgroup, 8 waves of 32, one workgroup a CU.  Every wave reads the same
// 64-key tiles of K and V in LDS, as bf16, four of each.  A wave takes its rows
// of a tile's codes into registers at the start of an iteration and converts
// them behind its products, so that K and V are converted once for all the
// queries: eight conversions of each for a lane's 32 logits.  (Codes copied to
// LDS first, three tiles ahead, with slots and scales in rings of their own:
// 286 us where this takes 270, 6044 rows of 32 heads over 2432 keys.)
// The loop is software pipelined: iteration t forms S(t + 1) while it
// exponentiates tile t's logits, then adds tile t's P V while it takes tile
// t + 1's maxima, and converts K(t + 3) and V(t + 2); a barrier at every second
// iteration orders that (at every one, with two tiles: 276).
// With 64-query waves or 128-query workgroups, two a CU, the registers do not
// suffice.  What remains between the loop and the matrix units' rate is spread
// over its parts: 182 us of products alone, 30 of exponentials, 23 and 17 of
// K and V fragment reads, 20 of conversions.
// ============================================================================
constexpr int kWdWaves = 8, kWdThreads = 64 * kWdWaves, kWdTileQ = 32 * kWdWaves;
constexpr int kWdKAhead = 4, kWdVAhead = 3;  // fragments read ahead of their product

__global__ __launch_bounds__(kWdThreads, 1) void quant_attention_wide_kernel(QAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char k_tile[4 * kTileB];
  __shared__ __attribute__((aligned(1024))) char v_tile[4 * kTileB];

  const Unit un = unit_of(a.rg, a.splits, (a.p.heads & 7) == 0 ? a.p.heads >> 3 : 1);
  const int g = un.g, b = un.b;
  const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nr = a.rg.cu_rows[b + 1] - a.rg.cu_rows[b];
  const int q0 = a.v_lo[b] + un.tile * kWdTileQ + wave * 32;
  const bool live = q0 < a.v_hi[b];  // wave-uniform: a wave without a query only copies and converts
  const int v = q0 + (lane & 31);
  const bool q_ok = v < a.v_hi[b];
  const int64_t pair = (int64_t)(a.rg.cu_rows[b] + (q_ok ? v % nr : 0)) * a.H + g * a.rep + (q_ok ? v / nr : 0);
  const int S = a.rg.cu_keys[b + 1] - a.rg.cu_keys[b];
  const int n_kt = (S + kTileK - 1) / kTileK;
  const int t_lo = (int)((int64_t)un.split * n_kt / a.splits), t_hi = (int)((int64_t)(un.split + 1) * n_kt / a.splits);
  const int key0 = t_lo * kTileK, n_keys = min(S, t_hi * kTileK) - key0;  // the workgroup's keys
  const int n_t = t_hi - t_lo;

  bf16x8 qf[8];
  load_query(a.q + pair * kDh, q_ok, hl, qf);

  const uint32_t n_slots = (uint32_t)a.p.n_slots;
  const uint32_t pool_b = (uint32_t)(a.p.n_slots * a.p.ld);  // < 2^31
  const uint32_t scale_b = (uint32_t)(((a.p.n_slots + (1 << a.p.shift) - 1) >> a.p.shift) * a.p.heads * 4);
  const auto kres = buffer_rsrc(a.p.codes[0], pool_b), vres = buffer_rsrc(a.p.codes[1], pool_b);
  const auto ksres = buffer_rsrc(a.p.scales[0], scale_b), vsres = buffer_rsrc(a.p.scales[1], scale_b);
  const auto sres = buffer_rsrc(a.slots + a.rg.cu_keys[b], (uint32_t)S * 4u);
  const uint32_t ld = (uint32_t)a.p.ld;

  // This wave's rows of a tile, one 16-byte chunk of codes a lane: row kk.
  // Tiles are counted from the first one.
  const int kk = wave * 8 + (lane >> 3), ch = lane & 7;
  struct Row {
    u32x4 codes;
    float scale;
  };
  struct Where {  // byte offsets of the row's codes and scale
    uint32_t code, scale;
  };
  auto load_slot = [&](int t) {
    return (int)__builtin_amdgcn_raw_buffer_load_b32(sres, (uint32_t)(key0 + t * kTileK + kk) * 4u, 0, 0);
  };
  auto locate = [&](int t, int slot) {
    const bool ok = t * kTileK + kk < n_keys && (uint32_t)slot < n_slots;
    return Where{ok ? (uint32_t)slot * ld + (uint32_t)g * kDh + ch * 16 : kAbsent,
                 ok ? (uint32_t)((slot >> a.p.shift) * a.p.heads + g) * 4u : kAbsent};
  };
  auto load_row = [](Where x, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t scales) {
    return Row{__builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, x.code, 0, 0)),
               __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(scales, x.scale, 0, 0))};
  };
  auto load_k = [&](Where x) { return load_row(x, kres, ksres); };
  auto load_v = [&](Where x) { return load_row(x, vres, vsres); };
  // Converted rows have 16-byte chunk c of row r at c ^ (r & 15) (K) and at
  // c ^ (4 (r & 3) ^ (r & 1)) (V): sixteen lanes' fragment reads and writes of
  // K, and 32 lanes' transposing reads of V (four rows of four chunks), then
  // cover all the banks.
  auto convert = [&](Row r, char* tile, int swizzle) {
    // an empty block's codes stand for zeros
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(r.scale > 0.f)) != 0, 0)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) r.codes[j] = r.scale > 0.f ? r.codes[j] : 0u;
    }
    u32x4 c[2];
    convert16(r.codes, r.scale, c);
    char* row = tile + kk * kRowB;
    *reinterpret_cast<u32x4*>(row + (((2 * ch) ^ swizzle) << 4)) = c[0];
    *reinterpret_cast<u32x4*>(row + (((2 * ch + 1) ^ swizzle) << 4)) = c[1];
  };
  auto convert_k = [&](int t, const Row& r) { convert(r, k_tile + (t & 3) * kTileB, kk & 15); };
  auto convert_v = [&](int t, const Row& r) { convert(r, v_tile + (t & 3) * kTileB, ((kk & 3) << 2) ^ (kk & 1)); };

  const float scale = kLog2e * rsqrtf((float)kDh);
  const int krow = key_perm(lane & 31);
  const int k_off = krow * kRowB, k_sw = krow & 15;  // the same swizzle for krow + 32
  const int vgrp = lane >> 4, gi = lane & 15;
  const int v_key = 8 * (vgrp >> 1) + (gi >> 2);
  const int v_chunk = 2 * (vgrp & 1) + ((gi & 3) >> 1);
  const int v_byte = (gi & 1) * 8, v_sw = (gi & 12) ^ ((gi >> 2) & 1);
  auto kfrag = [&](int t, int i) {
    const int kb = i >> 3, s = i & 7;
    return *reinterpret_cast<const bf16x8*>(k_tile + (t & 3) * kTileB + kb * 32 * kRowB + k_off +
                                            (((2 * s + hl) ^ k_sw) << 4));
  };
  auto vfrag = [&](int t, int i) {
    const int kb = i >> 3, g2 = (i >> 2) & 1, d = i & 3;
    const char* row = v_tile + (t & 3) * kTileB + (kb * 32 + g2 * 16 + v_key) * kRowB;
    const int off = ((4 * d + v_chunk) ^ v_sw) * 16 + v_byte;
    const v4i16 lo = ds_read_tr16(row + off);
    const v4i16 hi = ds_read_tr16(row + 4 * kRowB + off);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  f32x16 o_acc[4], st_a[2], st_b[2];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o_acc[d][r] = 0.f;
  float m_run = -INFINITY, l_part = 0.f;
  auto rescale = [&](float mx) {
    const bool bump = mx > m_run + 8.f;
    if (__builtin_amdgcn_ballot_w64(bump)) {
      const float alpha = bump ? __builtin_amdgcn_exp2f(m_run - mx) : 1.f;
      m_run = bump ? mx : m_run;
      l_part *= alpha;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[d][r] *= alpha;
    }
  };
  // the scaled maximum of a tile's logits, those of keys past the end made
  // -inf.  Register r of key block kb holds key 32 kb + 16 (r / 8) + 8 hl + r % 8.
  auto tile_max = [&](int t, f32x16 (&st)[2]) {
    const int n = n_keys - t * kTileK;  // > 0
    if (n < kTileK) {
      const uint64_t drop = ~0ull << n;
      const uint32_t dw[2] = {(uint32_t)drop >> (8 * hl), (uint32_t)(drop >> 32) >> (8 * hl)};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          st[kb][r] = (dw[kb] >> (16 * (r >> 3) + (r & 7))) & 1u ? -INFINITY : st[kb][r];
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kb][r]);
    return fmaxf(mx, __shfl_xor(mx, 32)) * scale;
  };

  int slot = 0;         // of tile t + 3 at iteration t
  Where v_at = {0, 0};  // of tile t + 2
  if (n_t > 0) {
    const int s0 = load_slot(0), s1 = load_slot(1), s2 = load_slot(2);
    slot = load_slot(3);
    const Where x0 = locate(0, s0), x1 = locate(1, s1);
    v_at = locate(2, s2);
    const Row k0 = load_k(x0), v0 = load_v(x0), k1 = load_k(x1), v1 = load_v(x1), k2 = load_k(v_at);
    convert_k(0, k0);
    convert_v(0, v0);
    convert_k(1, k1);
    convert_v(1, v1);
    convert_k(2, k2);
    wait_lgkmcnt<0>();
    bare_barrier();
    if (live) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) st_a[kb][r] = 0.f;
#pragma unroll
        for (int s = 0; s < 8; ++s) st_a[kb] = mfma32x32x16(kfrag(0, 8 * kb + s), qf[s], st_a[kb]);
      }
      rescale(tile_max(0, st_a));
    }
  }
  auto step = [&](int t, f32x16 (&cur)[2], f32x16 (&nxt)[2], bool sync) {
    // K to tile t + 2 and V to tile t + 1 are written, and what iterations t
    // and t + 1 write over has been read, by every wave
    if (sync) {
      wait_lgkmcnt<0>();
      bare_barrier();
    }
    __builtin_amdgcn_s_setprio(1);  // ahead of a wave that is between iterations
    const Where k_at = locate(t + 3, slot);
    const Row row_k = load_k(k_at), row_v = load_v(v_at);
    v_at = k_at;
    slot = load_slot(t + 4);
    if (!live) {
      __builtin_amdgcn_s_setprio(0);
      convert_k(t + 3, row_k);
      convert_v(t + 2, row_v);
      return;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    float psum = 0.f, mx = -INFINITY;
    bf16x8 pb[2][2];
    bf16x8 kf[kWdKAhead + 1], vf[kWdVAhead + 1];
    auto weight = [&](int e) {
      const int kb = e >> 4, r = e & 15;
      const float x = __builtin_amdgcn_exp2f(fmaf(cur[kb][r], scale, -m_use));
      psum += x;
      pb[kb][r >> 3][r & 7] = (bf16)x;
    };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) nxt[kb][r] = 0.f;
#pragma unroll
    for (int i = 0; i < kWdKAhead; ++i) kf[i] = kfrag(t + 1, i);
    // sixteen products of S(t + 1), each with an exponential of tile t, then
    // sixteen of P V: the first eight with two exponentials each, the others
    // with the maxima of four of tile t + 1's logits.  The empty asm statements
    // keep the running sum and maximum in their place.
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + kWdKAhead < 16) kf[(i + kWdKAhead) % (kWdKAhead + 1)] = kfrag(t + 1, i + kWdKAhead);
      if (i >= 16 - kWdVAhead) vf[i - (16 - kWdVAhead)] = vfrag(t, i - (16 - kWdVAhead));
      nxt[i >> 3] = mfma32x32x16(kf[i % (kWdKAhead + 1)], qf[i & 7], nxt[i >> 3]);
      weight(i);
      asm volatile("" ::"v"(psum));
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + kWdVAhead < 16) vf[(i + kWdVAhead) % (kWdVAhead + 1)] = vfrag(t, i + kWdVAhead);
      o_acc[i & 3] = mfma32x32x16(vf[i % (kWdVAhead + 1)], pb[i >> 3][(i >> 2) & 1], o_acc[i & 3]);
      if (i < 8) {
        weight(16 + 2 * i);
        weight(17 + 2 * i);
        asm volatile("" ::"v"(psum));
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) mx = fmaxf(mx, nxt[(i - 8) >> 2][4 * (i & 3) + u]);
        asm volatile("" ::"v"(mx));
      }
      if (i == 10) convert_k(t + 3, row_k);
      if (i == 13) convert_v(t + 2, row_v);
      __builtin_amdgcn_sched_barrier(0);
    }
    l_part += psum;
    __builtin_amdgcn_s_setprio(0);
    if (t + 1 < n_t) {
      if ((t + 2) * kTileK > n_keys) mx = tile_max(t + 1, nxt);
      else mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
      rescale(mx);
    }
  };
  for (int t = 0; t < n_t; t += 4) {
    step(t, st_a, st_b, true);
    if (t + 1 < n_t) step(t + 1, st_b, st_a, false);
    if (t + 2 < n_t) step(t + 2, st_a, st_b, true);
    if (t + 3 < n_t) step(t + 3, st_b, st_a, false);
  }

  if (!live) return;
  const float l_tot = l_part + __shfl_xor(l_part, 32);
  if (q_ok) write_query(a, pair, un.split, hl, o_acc, m_run, l_tot);
}

// ============================================================================
// quant_attention_narrow_kernel: 32 queries of one KV head and request, the
// keys dealt to the four waves of a workgroup, which never wait for each other
// until their results are combined: for calls with few queries, whose time is
// reading the cache.
// A wave reads 32-key tiles of codes two tiles ahead into registers (a lane
// 16 bytes, eight lanes a row, which is what the address path is fast for),
// and passes them through LDS of its own to the operands' layouts, still as
// codes.  They are converted in registers: K by rows, times its scale, lane
// half hl supplying dimensions 64 hl + 8 s .. + 7 to product s and the query
// held in the same order; V by a transposing read of bytes (in each 16-lane
// group lane i points at key i / 2, dimensions 8 (i % 2) .. + 7 and receives
// dimension i of the 8 keys), unscaled, the scale being a factor of the weight
// instead (which below 2^-126, a small weight at one of the smallest scales, is a
// subnormal bf16: the product takes it, off by at most 2^-134, so an output by
// at most 448 * 2^-134 for each key).  16-byte chunk c of row r lies at c ^ k_swizzle(r) (K) and
// c ^ (r & 7) (V).  Slots are read and offsets and scales made for 64 keys at a
// time, one key a lane.
// Measured: keys that one request alone reads at 5.1 TB/s, the rate of a large
// copy, with all CUs busy (a query of 8 requests over 30,000 keys of 4 heads:
// 48 us); keys that lie in the caches 0.95 us a tile of 32 for a wave, which is
// its conversions, products and weights one after the other.  32 rows of each
// of 32 requests, 32 heads, over 8704 keys take 233 us; with codes copied
// straight to LDS 247, with the loop software pipelined 238, with neighbouring
// heads side by side in the grid 281.
// ============================================================================
constexpr int kNwWaves = 4;
constexpr int kNwTileK = 32;
constexpr int kNwTileB = kNwTileK * kDh;   // 4 KB of codes
constexpr int kNwCopies = kNwTileB / 1024;
constexpr int kNwWaveB = 2 * kNwTileB + 4 * kAuxB;  // a wave's LDS
static_assert(kNwWaves * kNwWaveB >= 2 * 66 * 64 * 4, "room for two waves' results");

// Between LDS writes of a wave's lanes and reads of what other lanes wrote, and
// between such reads and the next writes: the LDS keeps a wave's order by
// itself (nothing is waited for), and this makes the compiler keep it, which
// sees one lane's addresses only.
__device__ __forceinline__ void lane_handoff() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}
__device__ __forceinline__ int k_swizzle(int r) { return (r & 3) | ((r >> 1) & 4); }
__device__ __forceinline__ bf16x8 v_fragment(const char* lds) {
  typedef int v2i32 __attribute__((__vector_size__(2 * sizeof(int))));
  const v2i32 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i32*)lds);
  u32x4 c;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    c[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, false));
    c[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, true));
  }
  return __builtin_bit_cast(bf16x8, c);
}

__global__ __launch_bounds__(64 * kNwWaves, 2) void quant_attention_narrow_kernel(QAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[kNwWaves * kNwWaveB];

  const Unit un = unit_of(a.rg, a.splits, 1);
  const int g = un.g, b = un.b;
  const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5, row = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nr = a.rg.cu_rows[b + 1] - a.rg.cu_rows[b];
  const int v = a.v_lo[b] + un.tile * 32 + row;
  const bool q_ok = v < a.v_hi[b];
  const int64_t pair = (int64_t)(a.rg.cu_rows[b] + (q_ok ? v % nr : 0)) * a.H + g * a.rep + (q_ok ? v / nr : 0);
  const int S = a.rg.cu_keys[b + 1] - a.rg.cu_keys[b];
  const int n_kt = (S + kNwTileK - 1) / kNwTileK;
  const int parts = a.splits * kNwWaves, part = un.split * kNwWaves + wave;
  const int t_lo = (int)((int64_t)part * n_kt / parts), t_hi = (int)((int64_t)(part + 1) * n_kt / parts);
  const int key0 = t_lo * kNwTileK, n_keys = min(S, t_hi * kNwTileK) - key0;  // this wave's keys
  const int n_t = t_hi - t_lo;

  bf16x8 qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (q_ok) w = *reinterpret_cast<const u32x4*>(a.q + pair * kDh + 64 * hl + 8 * s);
    qf[s] = __builtin_bit_cast(bf16x8, w);
  }

  const uint32_t n_slots = (uint32_t)a.p.n_slots;
  const uint32_t pool_b = (uint32_t)(a.p.n_slots * a.p.ld);  // < 2^31
  const uint32_t scale_b = (uint32_t)(((a.p.n_slots + (1 << a.p.shift) - 1) >> a.p.shift) * a.p.heads * 4);
  const auto kres = buffer_rsrc(a.p.codes[0], pool_b), vres = buffer_rsrc(a.p.codes[1], pool_b);
  const auto ksres = buffer_rsrc(a.p.scales[0], scale_b), vsres = buffer_rsrc(a.p.scales[1], scale_b);
  const auto sres = buffer_rsrc(a.slots + a.rg.cu_keys[b], (uint32_t)S * 4u);

  // Tiles and 64-key groups are counted from this wave's first key.  In LDS: a
  // tile of K and of V codes, byte offsets of two groups, scales of one.
  char* const kt = lds + wave * kNwWaveB;
  char* const vt = kt + kNwTileB;
  char* const offsets = vt + kNwTileB;
  char* const k_scales = offsets + 2 * kAuxB;
  char* const v_scales = k_scales + kAuxB;
  struct Scales {
    uint32_t k, v;
  };
  auto load_slot = [&](int u) {
    return (int)__builtin_amdgcn_raw_buffer_load_b32(sres, (uint32_t)(key0 + u * 64 + lane) * 4u, 0, 0);
  };
  auto has_key = [&](int u, int slot) { return u * 64 + lane < n_keys && (uint32_t)slot < n_slots; };
  auto put_offset = [&](int u, int slot) {
    const uint32_t off = (uint32_t)slot * (uint32_t)a.p.ld + (uint32_t)g * kDh;
    *reinterpret_cast<uint32_t*>(offsets + (u & 1) * kAuxB + lane * 4) = has_key(u, slot) ? off : kAbsent;
  };
  auto load_scales = [&](int u, int slot, Scales& x) {
    const uint32_t off = has_key(u, slot) ? (uint32_t)((slot >> a.p.shift) * a.p.heads + g) * 4u : kAbsent;
    x.k = __builtin_amdgcn_raw_buffer_load_b32(ksres, off, 0, 0);
    x.v = __builtin_amdgcn_raw_buffer_load_b32(vsres, off, 0, 0);
  };
  auto put_scales = [&](const Scales& x) {
    *reinterpret_cast<float*>(k_scales + lane * 4) = __uint_as_float(x.k);  // its readers' type
    *reinterpret_cast<float*>(v_scales + lane * 4) = pow2_below(__uint_as_float(x.v));
    return __builtin_amdgcn_ballot_w64(!(__uint_as_float(x.k) > 0.f) || !(__uint_as_float(x.v) > 0.f)) != 0;
  };
  const int lrow = lane >> 3, lch = lane & 7;
  struct Codes {
    u32x4 k[kNwCopies], v[kNwCopies];
  };
  auto load_codes = [&](int t, Codes& x) {
#pragma unroll
    for (int i = 0; i < kNwCopies; ++i) {
      const uint32_t off =
          *reinterpret_cast<const uint32_t*>(offsets + ((t >> 1) & 1) * kAuxB + ((t & 1) * kNwTileK + 8 * i + lrow) * 4) +
          lch * 16;
      x.k[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kres, off, 0, 0));
      x.v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vres, off, 0, 0));
    }
  };
  auto put_codes = [&](int t, Codes& x, bool empty) {
    if (empty) {  // an empty block's codes stand for zeros
      lane_handoff();
#pragma unroll
      for (int i = 0; i < kNwCopies; ++i) {
        const int at = ((t & 1) * kNwTileK + 8 * i + lrow) * 4;
        const bool ke = *reinterpret_cast<const float*>(k_scales + at) > 0.f;
        const bool ve = *reinterpret_cast<const float*>(v_scales + at) > 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x.k[i][j] = ke ? x.k[i][j] : 0u;
          x.v[i][j] = ve ? x.v[i][j] : 0u;
        }
      }
      lane_handoff();
    }
#pragma unroll
    for (int i = 0; i < kNwCopies; ++i) {
      const int r = 8 * i + lrow;
      *reinterpret_cast<u32x4*>(kt + r * kDh + ((lch ^ k_swizzle(r)) << 4)) = x.k[i];
      *reinterpret_cast<u32x4*>(vt + r * kDh + ((lch ^ (r & 7)) << 4)) = x.v[i];
    }
  };

  const float scale = kLog2e * rsqrtf((float)kDh);
  const int krow = key_perm(row), k_sw = k_swizzle(krow);
  const int vgrp = lane >> 4, gi = lane & 15;
  const int v_key = 8 * (vgrp >> 1) + (gi >> 1);
  const int v_off = v_key * kDh + (gi & 1) * 8, v_sw = v_key & 7, v_ch = vgrp & 1;

  f32x16 o_acc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o_acc[d][r] = 0.f;
  float m_run = -INFINITY, l_part = 0.f;

  auto step = [&](int t) {
    const float ks = *reinterpret_cast<const float*>(k_scales + ((t & 1) * kNwTileK + krow) * 4);
    f32x16 st;
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(kt + krow * kDh + (((4 * hl + i) ^ k_sw) << 4));
      u32x4 c[2];
      convert16(w, ks, c);
      st = mfma32x32x16(__builtin_bit_cast(bf16x8, c[0]), qf[2 * i], st);
      st = mfma32x32x16(__builtin_bit_cast(bf16x8, c[1]), qf[2 * i + 1], st);
    }
    // register r holds key 16 (r / 8) + 8 hl + r % 8
    const int n = n_keys - t * kNwTileK;  // > 0
    if (n < kNwTileK) {
      const uint32_t drop = (~0u << n) >> (8 * hl);
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = (drop >> (16 * (r >> 3) + (r & 7))) & 1u ? -INFINITY : st[r];
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
    const bool bump = mx > m_run + 8.f;
    if (__builtin_amdgcn_ballot_w64(bump)) {
      const float alpha = bump ? __builtin_amdgcn_exp2f(m_run - mx) : 1.f;
      m_run = bump ? mx : m_run;
      l_part *= alpha;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[d][r] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    const char* vs = v_scales + ((t & 1) * kNwTileK + 8 * hl) * 4;
    bf16x8 pb[2];
#pragma unroll
    for (int g2 = 0; g2 < 2; ++g2) {
      f32x4 sv[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) sv[j] = *reinterpret_cast<const f32x4*>(vs + (16 * g2 + 4 * j) * 4);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = __builtin_amdgcn_exp2f(fmaf(st[8 * g2 + j], scale, -m_use));
        l_part += e;
        pb[g2][j] = (bf16)(e * sv[j >> 2][j & 3]);
      }
    }
#pragma unroll
    for (int g2 = 0; g2 < 2; ++g2)
#pragma unroll
      for (int d = 0; d < 4; ++d)
        o_acc[d] = mfma32x32x16(v_fragment(vt + 16 * g2 * kDh + v_off + (((2 * d + v_ch) ^ v_sw) << 4)), pb[g2],
                                o_acc[d]);
  };

  if (n_t > 0) {
    Codes x0, x1;
    Scales sa, sb;
    const int s0 = load_slot(0), s1 = load_slot(1);
    int next = load_slot(2);
    put_offset(0, s0);
    put_offset(1, s1);
    lane_handoff();
    load_codes(0, x0);
    load_codes(1, x1);
    load_scales(0, s0, sa);
    load_scales(1, s1, sb);
    for (int t = 0; t < n_t; t += 2) {
      const int u = t >> 1;
      lane_handoff();
      const bool empty = put_scales(sa);
      put_codes(t, x0, empty);
      lane_handoff();
      load_codes(t + 2, x0);
      step(t);
      lane_handoff();
      put_codes(t + 1, x1, empty);
      put_offset(u + 2, next);  // over group u's
      lane_handoff();
      load_codes(t + 3, x1);
      sa = sb;
      load_scales(u + 2, next, sb);
      next = load_slot(u + 3);
      if (t + 1 < n_t) step(t + 1);
    }
  }

  // the waves' results, lane by lane: 1 into 0 and 3 into 2, then 2 into 0
  float l = l_part + __shfl_xor(l_part, 32), m = m_run;
#pragma unroll
  for (int round = 0; round < 2; ++round) {
    const bool give = round == 0 ? (wave & 1) : wave == 2, take = round == 0 ? !(wave & 1) : wave == 0;
    f32x4* const o_at = reinterpret_cast<f32x4*>(lds + (round == 0 ? wave >> 1 : 0) * (66 * 64 * 4)) + lane;
    float2* const ml_at = reinterpret_cast<float2*>(o_at - lane + 16 * 64) + lane;
    __syncthreads();
    if (give) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        o_at[i * 64] = f32x4{o_acc[i >> 2][4 * (i & 3)], o_acc[i >> 2][4 * (i & 3) + 1], o_acc[i >> 2][4 * (i & 3) + 2],
                             o_acc[i >> 2][4 * (i & 3) + 3]};
      *ml_at = float2{m, l};
    }
    __syncthreads();
    if (take) {
      const float2 ml = *ml_at;
      const float mn = fmaxf(m, ml.x);
      const float f0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      const float f1 = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mn);
      l = l * f0 + ml.y * f1;
      m = mn;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const f32x4 o = o_at[i * 64];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o_acc[i >> 2][4 * (i & 3) + j] = o_acc[i >> 2][4 * (i & 3) + j] * f0 + o[j] * f1;
      }
    }
  }
  if (wave == 0 && q_ok) write_query(a, pair, un.split, hl, o_acc, m, l);
}

// Combines the key splits of each (row, head): m = max_s m_s, O = sum_s
// 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  A wave per (row, head): lane s holds
// split s's max and sum; lane half hf sums 4 dimensions a lane over the splits
// s with (s / 8) % 2 == hf, in order, eight loads in flight at a time (a chain
// of loads is what bounds it), and the halves are added last.  1024 pairs of six
// splits add 2.5 us to the call (4 with a load at a time).
__global__ __launch_bounds__(256) void quant_attention_merge_kernel(const float* __restrict__ part_o,
                                                                    const float* __restrict__ part_ml, int splits,
                                                                    int64_t pairs, bf16* __restrict__ out,
                                                                    float* __restrict__ lse) {
  const int64_t pair = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (pair >= pairs) return;
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  float2 ml = {-INFINITY, 0.f};
  if (lane < splits) ml = *reinterpret_cast<const float2*>(part_ml + (lane * pairs + pair) * 2);
  const float* po = part_o + pair * kDh + (lane & 31) * 4;
  float w = 0.f, m = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += 16) {
    f32x4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = s0 + 8 * hf + i;
      v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (s < splits) v[i] = *reinterpret_cast<const f32x4*>(po + s * pairs * kDh);
    }
    if (s0 == 0) {  // behind the first loads
      m = wave_max(ml.x);
      w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float ws = __shfl(w, (s0 + 8 * hf + i) & 63);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += ws * v[i][j];
    }
  }
  const float l = wave_sum(w * ml.y);
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], 32);
  if (hf) return;
  const float inv = 1.f / l;
  bf16x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (bf16)(o[j] * inv);
  *reinterpret_cast<bf16x4*>(out + pair * kDh + lane * 4) = r;
  if (lse && lane == 0) lse[pair] = (m + __log2f(l)) * kLn2;
}

}  // namespace

// Partials of `pairs` (row, head) pairs: as many splits as keep the splits of
// all pairs within kPartPairs, so that a workspace serves every smaller call.
constexpr int64_t kPartPairs = 65536;
size_t quant_attention_part_bytes(int64_t pairs) {
  return (size_t)std::min<int64_t>(kPartPairs, pairs * kMaxSplits) * (kDh + 2) * sizeof(float);
}

namespace {

// Estimated time (us) of `units` (query tile, KV head) pairs over n_kt 64-key
// tiles and the key splits that give it, within `fit`.  Measured: a launch and
// its first loads 6, 7.5 with two workgroups on a CU; a step of the narrow
// kernel (32 keys a wave) 0.95, or 1.65 with two workgroups on a CU; a tile of
// the wide kernel 1.9, one workgroup a CU; a merge 3.5 and its partials at 3
// TB/s.  memory_us: the keys at 4.9 TB/s on all CUs, each request's read once,
// which is what keys of a request's own cost at least; keys that requests share
// come from the caches after the first and cost less than it says (32 requests
// over a shared affix of 8192 keys and 512 of their own: 465 us, where the call
// takes 235): there the estimate can leave splits unused.
// Both sides of the choice, in us, narrow and wide at their best splits:
//   32 rows, 32 heads, 1536 keys  11.6 / 12.0;  717 rows  38 / 41
//   8 x 512 rows, 32 heads, 2432 keys  273 / 168
//   4 x 32 rows, 28 heads on 4, 5120 keys  29.5 / 29.6;  4 x 256 rows  122 / 89
struct Cost {
  double us;
  int splits;
};
double merge_us(int splits, int64_t pairs) {
  return splits > 1 ? 3.5 + 2.0 * splits * pairs * (kDh + 2) * sizeof(float) / 3e6 : 0.0;
}
Cost narrow_cost(int64_t units, int n_kt, double memory_us, int64_t pairs, int64_t fit) {
  Cost best = {1e30, 1};
  for (int s = 1; s <= std::min<int64_t>(fit, kMaxSplits); ++s) {
    const int64_t wgs = units * s, rest = wgs % 512;
    const int steps = (2 * n_kt + kNwWaves * s - 1) / (kNwWaves * s);
    const double loop = steps * (1.65 * (wgs / 512) + (rest == 0 ? 0.0 : rest <= 256 ? 0.95 : 1.65));
    const double memory = memory_us * 256.0 / std::min<int64_t>(wgs, 256);
    const double us = (wgs <= 256 ? 6.0 : 7.5) + std::max(loop, memory) + merge_us(s, pairs);
    if (us < best.us) best = {us, s};
    if (steps == 1) break;
  }
  return best;
}
Cost wide_cost(int64_t units, int n_kt, double memory_us, int64_t pairs, int64_t fit) {
  Cost best = {1e30, 1};
  for (int s = 1; s <= std::min<int64_t>(std::min<int64_t>(fit, kMaxSplits), std::max(n_kt, 1)); ++s) {
    const double loop = 1.9 * ((n_kt + s - 1) / s) * (double)((units * s + 255) / 256);
    const double memory = memory_us * 256.0 / std::min<int64_t>(units * s, 256);
    const double us = 6.0 + std::max(loop, memory) + merge_us(s, pairs);
    if (us < best.us) best = {us, s};
  }
  return best;
}

}  // namespace

QuantAttentionPlan plan_quant_attention(const Ragged& rg, int H, int kv_heads, size_t part_bytes) {
  const int64_t pairs = (int64_t)rg.cu_rows[rg.batch] * H;
  QuantAttentionPlan plan = {0, 0, 0, 1};
  if (pairs == 0) return plan;
  // query tiles of each kernel, and of the wide kernel with the narrow one
  // behind it on what is left of a request behind its whole tiles, where that
  // is at most kRest[i] queries
  constexpr int kRest[3] = {64, 128, kWdTileQ - 1};
  int64_t narrow = 0, wide = 0, both_wide[3] = {}, both_narrow[3] = {};
  int n_kt = 0;
  double memory_us = 0.0;
  for (int b = 0; b < rg.batch; ++b) {
    const int64_t n = (int64_t)(rg.cu_rows[b + 1] - rg.cu_rows[b]) * (H / kv_heads);
    narrow += (n + 31) / 32;
    wide += (n + kWdTileQ - 1) / kWdTileQ;
    for (int i = 0; i < 3; ++i) {
      const bool few = n % kWdTileQ <= kRest[i];
      both_wide[i] += few ? n / kWdTileQ : (n + kWdTileQ - 1) / kWdTileQ;
      both_narrow[i] += few ? (n % kWdTileQ + 31) / 32 : 0;
    }
    n_kt = std::max(n_kt, (rg.cu_keys[b + 1] - rg.cu_keys[b] + kTileK - 1) / kTileK);
    if (n > 0) memory_us += (rg.cu_keys[b + 1] - rg.cu_keys[b]) * (2.0 * kDh / 4.9e6) * kv_heads;
  }
  const int64_t fit = std::max<int64_t>(1, (int64_t)(part_bytes / ((kDh + 2) * sizeof(float))) / pairs);
  const Cost cn = narrow_cost(narrow * kv_heads, n_kt, memory_us, pairs, fit);
  const Cost cw = wide_cost(wide * kv_heads, n_kt, memory_us, pairs, fit);
  // the two launches write no partials: a merge would cover every row
  double both_us = 1e30;
  int both = 0;
  for (int i = 0; i < 3; ++i) {
    if (!both_wide[i] || !both_narrow[i]) continue;
    const double us = wide_cost(both_wide[i] * kv_heads, n_kt, memory_us, pairs, 1).us +
                      narrow_cost(both_narrow[i] * kv_heads, n_kt, 0.0, pairs, 1).us;
    if (us < both_us) both_us = us, both = i;
  }
  if (both_us < std::min(cn.us, cw.us)) plan = {(int)both_wide[both], (int)both_narrow[both], kRest[both], 1};
  else if (cw.us < cn.us) plan = {(int)wide, 0, 0, cw.splits};
  else plan = {0, (int)narrow, 0, cn.splits};
  return plan;
}

hipError_t launch_quant_attention(const Ragged& rg, int H, const QuantPool& p, const void* q, const int32_t* read_slots,
                                  void* out, float* lse, float* part, size_t part_bytes, hipStream_t s) {
  const int64_t pairs = (int64_t)rg.cu_rows[rg.batch] * H;
  if (pairs == 0) return hipSuccess;
  const QuantAttentionPlan plan = plan_quant_attention(rg, H, p.heads, part_bytes);
  const int splits = plan.splits;
  QAttnArgs a;
  a.p = p;
  a.q = (const bf16*)q;
  a.slots = read_slots;
  a.out = (bf16*)out;
  a.lse = lse;
  a.H = H;
  a.rep = H / p.heads;
  a.rg = rg;
  a.splits = splits;
  a.part_o = part;
  a.part_ml = part ? part + (size_t)splits * pairs * kDh : nullptr;
  // one launch over each request's queries: all of them, or those left to (or
  // by) the other kernel
  auto launch = [&](bool is_wide) {
    const bool share = plan.wide_tiles && plan.narrow_tiles;
    const int tq = is_wide ? kWdTileQ : 32;
    int tiles = 0;
    for (int b = 0; b < rg.batch; ++b) {
      const int n = (rg.cu_rows[b + 1] - rg.cu_rows[b]) * a.rep;
      const int cut = n % kWdTileQ <= plan.rest ? n - n % kWdTileQ : n;
      a.rg.tile_start[b] = tiles;
      a.v_lo[b] = share && !is_wide ? cut : 0;
      a.v_hi[b] = share && is_wide ? cut : n;
      tiles += (a.v_hi[b] - a.v_lo[b] + tq - 1) / tq;
    }
    a.rg.tile_start[rg.batch] = tiles;
    const dim3 grid((unsigned)((int64_t)tiles * p.heads * splits));
    if (is_wide) hipLaunchKernelGGL(quant_attention_wide_kernel, grid, dim3(kWdThreads), 0, s, a);
    else hipLaunchKernelGGL(quant_attention_narrow_kernel, grid, dim3(64 * kNwWaves), 0, s, a);
  };
  if (plan.wide_tiles) launch(true);
  if (plan.narrow_tiles) launch(false);
  if (splits > 1)
    hipLaunchKernelGGL(quant_attention_merge_kernel, dim3((unsigned)((pairs + 3) / 4)), dim3(256), 0, s,
                       (const float*)a.part_o, (const float*)a.part_ml, splits, pairs, a.out, lse);
  return hipGetLastError();
}

}  // namespace acache
