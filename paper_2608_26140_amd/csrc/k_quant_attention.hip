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
// the product with V, as in the bf16 attention.
//
// With grouped heads the query heads of a KV head are further queries of the
// same tile: a request's query v is row v mod rows of head g rep + v / rows.
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
constexpr int kCodeTileB = kTileK * kDh;      // 8 KB: the codes of one K or V tile
constexpr int kRowB = kDh * 2;                // a converted row
constexpr int kTileB = kTileK * kRowB;        // 16 KB: a converted tile
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
  Ragged rg;       // tile_start: query tiles of a KV head
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

// The (KV head, request, query tile, key split) of a workgroup: KV heads
// outermost and XCD-contiguous, so that workgroups that share keys share an L2.
struct Unit {
  int g, b, tile, split;
};
__device__ __forceinline__ Unit unit_of(const Ragged& rg, int splits) {
  const int n_tiles = rg.tile_start[rg.batch];
  const int nb = gridDim.x, i = blockIdx.x;
  const int q8 = nb >> 3, r8 = nb & 7, x = i & 7;
  const int t = x * q8 + min(x, r8) + (i >> 3);
  Unit u;
  u.g = t / (n_tiles * splits);
  const int rem = t - u.g * n_tiles * splits;
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
// workgroup, 8 waves of 32.  Every wave reads the same 64-key tiles: the codes
// of K and V come to LDS by buffer copies some tiles ahead (issued from inline
// assembly, which the compiler's wait analysis does not drain, and waited for
// by counting), the slots and scales that the copies' addresses need earlier
// still, by waves 0, 1 and 2.  Each wave converts the rows it copied to bf16
// one iteration ahead of their use: eight conversions of K and of V for a
// lane's 32 logits.
// The loop is software pipelined: iteration t forms S(t + 1) while it
// exponentiates tile t's logits, then adds tile t's P V while it takes tile
// t + 1's maxima, and converts K(t + 2) and V(t + 1).
// ============================================================================
constexpr int kWdWaves = 8;
constexpr int kWdThreads = 64 * kWdWaves;
constexpr int kWdTileQ = 32 * kWdWaves;
constexpr int kWdStages = 4;  // rings of K and V codes
constexpr int kWdAux = 8;     // rings of slots and scales
constexpr int kAuxB = kTileK * 4;
constexpr int kWdKAhead = 3, kWdVAhead = 2;  // fragments read ahead of their product

__global__ __launch_bounds__(kWdThreads, 1) void quant_attention_wide_kernel(QAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char k_codes[kWdStages * kCodeTileB];
  __shared__ __attribute__((aligned(1024))) char v_codes[kWdStages * kCodeTileB];
  __shared__ __attribute__((aligned(1024))) char k_tile[2 * kTileB];
  __shared__ __attribute__((aligned(1024))) char v_tile[2 * kTileB];
  __shared__ __attribute__((aligned(256))) char slot_ring[kWdAux * kAuxB];
  __shared__ __attribute__((aligned(256))) char ks_ring[kWdAux * kAuxB];
  __shared__ __attribute__((aligned(256))) char vs_ring[kWdAux * kAuxB];

  const Unit un = unit_of(a.rg, a.splits);
  const int g = un.g, b = un.b;
  const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nr = a.rg.cu_rows[b + 1] - a.rg.cu_rows[b];
  const int q0 = un.tile * kWdTileQ + wave * 32;
  const bool live = q0 < nr * a.rep;  // wave-uniform: a wave without a query only copies and converts
  const int v = q0 + (lane & 31);
  const bool q_ok = v < nr * a.rep;
  const int64_t pair = (int64_t)(a.rg.cu_rows[b] + (q_ok ? v % nr : 0)) * a.H + g * a.rep + (q_ok ? v / nr : 0);
  const int S = a.rg.cu_keys[b + 1] - a.rg.cu_keys[b];
  const int n_kt = (S + kTileK - 1) / kTileK;
  const int t_lo = (int)((int64_t)un.split * n_kt / a.splits), t_hi = (int)((int64_t)(un.split + 1) * n_kt / a.splits);
  const int key_end = min(S, t_hi * kTileK);  // the workgroup's keys end here

  bf16x8 qf[8];
  load_query(a.q + pair * kDh, q_ok, hl, qf);

  const uint32_t pool_b = (uint32_t)(a.p.n_slots * a.p.ld);  // < 2^31
  const uint32_t scale_b = (uint32_t)(((a.p.n_slots + (1 << a.p.shift) - 1) >> a.p.shift) * a.p.heads * 4);
  const rsrc_words kres = buffer_words(a.p.codes[0], pool_b), vres = buffer_words(a.p.codes[1], pool_b);
  const rsrc_words ksres = buffer_words(a.p.scales[0], scale_b), vsres = buffer_words(a.p.scales[1], scale_b);
  const rsrc_words sres = buffer_words(a.slots + a.rg.cu_keys[b], (uint32_t)S * 4u);
  const uint32_t ld = (uint32_t)a.p.ld;

  auto aux = [](char* ring, int t) { return ring + (t & (kWdAux - 1)) * kAuxB; };
  auto issue_slots = [&](int t) { dma4_asm(sres, (uint32_t)(t * kTileK + lane) * 4u, aux(slot_ring, t)); };
  // the scales of tile t's keys; 0, an empty block's, where there is no key or no such slot
  auto issue_scales = [&](int t, rsrc_words res, char* ring) {
    const int slot = *reinterpret_cast<const int*>(aux(slot_ring, t) + lane * 4);
    const bool ok = t * kTileK + lane < key_end && slot >= 0 && slot < a.p.n_slots;
    dma4_asm(res, ok ? (uint32_t)((slot >> a.p.shift) * a.p.heads + g) * 4u : kAbsent, aux(ring, t));
  };
  auto issue_aux = [&](int t_slots) {
    if (wave == 0) issue_slots(t_slots);
    if (wave == 1) issue_scales(t_slots - 1, ksres, ks_ring);
    if (wave == 2) issue_scales(t_slots - 1, vsres, vs_ring);
  };
  // This wave's rows of a tile, one 16-byte chunk of codes a lane: row kk.  Of
  // an empty block the copies give zeros.
  const int kk = wave * 8 + (lane >> 3), ch = lane & 7;
  auto issue_codes = [&](int t, rsrc_words res, char* ring, char* scales) {
    const int slot = *reinterpret_cast<const int*>(aux(slot_ring, t) + kk * 4);
    const float sc = *reinterpret_cast<const float*>(aux(scales, t) + kk * 4);
    const uint32_t off = (uint32_t)slot * ld + (uint32_t)g * kDh + ch * 16;
    dma16_asm(res, sc > 0.f ? off : kAbsent, ring + (t & (kWdStages - 1)) * kCodeTileB + wave * 1024);
  };
  // Converted rows have 16-byte chunk c of row r at c ^ (r & 15) (K) and at
  // c ^ 2 (r & 3) (V), as their fragment reads need it.
  auto convert = [&](int t, const char* ring, char* scales, char* tile, int swizzle) {
    const float sc = *reinterpret_cast<const float*>(aux(scales, t) + kk * 4);
    const u32x4 w =
        *reinterpret_cast<const u32x4*>(ring + (t & (kWdStages - 1)) * kCodeTileB + wave * 1024 + lane * 16);
    u32x4 c[2];
    convert16(w, sc, c);
    char* row = tile + (t & 1) * kTileB + kk * kRowB;
    *reinterpret_cast<u32x4*>(row + (((2 * ch) ^ swizzle) << 4)) = c[0];
    *reinterpret_cast<u32x4*>(row + (((2 * ch + 1) ^ swizzle) << 4)) = c[1];
  };
  auto convert_k = [&](int t) { convert(t, k_codes, ks_ring, k_tile, kk & 15); };
  auto convert_v = [&](int t) { convert(t, v_codes, vs_ring, v_tile, (kk & 3) << 1); };

  const float scale = kLog2e * rsqrtf((float)kDh);
  const int krow = key_perm(lane & 31);
  const int k_off = krow * kRowB, k_sw = krow & 15;  // the same swizzle for krow + 32
  const int vgrp = lane >> 4, gi = lane & 15;
  const int v_key = 8 * (vgrp >> 1) + (gi >> 2);
  const int v_chunk = 2 * (vgrp & 1) + ((gi & 3) >> 1);
  const int v_byte = (gi & 1) * 8, v_sw = (gi >> 2) << 1;
  auto kfrag = [&](int t, int i) {
    const int kb = i >> 3, s = i & 7;
    return *reinterpret_cast<const bf16x8*>(k_tile + (t & 1) * kTileB + kb * 32 * kRowB + k_off +
                                            (((2 * s + hl) ^ k_sw) << 4));
  };
  auto vfrag = [&](int t, int i) {
    const int kb = i >> 3, g2 = (i >> 2) & 1, d = i & 3;
    const char* row = v_tile + (t & 1) * kTileB + (kb * 32 + g2 * 16 + v_key) * kRowB;
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
    const int n = key_end - t * kTileK;  // > 0
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

  if (t_lo < t_hi) {
    // prologue: the slots of six tiles, the scales of five, the codes of four
    // K tiles and three V tiles
    if (wave == 0)
      for (int i = 0; i < 6; ++i) issue_slots(t_lo + i);
    wait_vm_asm<0>();
    bare_barrier();
    if (wave == 1)
      for (int i = 0; i < 5; ++i) issue_scales(t_lo + i, ksres, ks_ring);
    if (wave == 2)
      for (int i = 0; i < 5; ++i) issue_scales(t_lo + i, vsres, vs_ring);
    wait_vm_asm<0>();
    bare_barrier();
    issue_codes(t_lo, kres, k_codes, ks_ring);
    for (int i = 0; i < 3; ++i) {
      issue_codes(t_lo + i + 1, kres, k_codes, ks_ring);
      issue_codes(t_lo + i, vres, v_codes, vs_ring);
    }
    wait_vm_asm<4>();  // K of two tiles, V of one
    convert_k(t_lo);
    convert_k(t_lo + 1);
    convert_v(t_lo);
    wait_lgkmcnt<0>();
    bare_barrier();
    if (live) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) st_a[kb][r] = 0.f;
#pragma unroll
        for (int s = 0; s < 8; ++s) st_a[kb] = mfma32x32x16(kfrag(t_lo, 8 * kb + s), qf[s], st_a[kb]);
      }
      rescale(tile_max(t_lo, st_a));
    }
  }
  auto step = [&](int t, f32x16 (&cur)[2], f32x16 (&nxt)[2]) {
    // all but the last iteration's two copies of codes have landed: K codes up
    // to t + 2, V codes to t + 1, scales to t + 4, slots to t + 5; and what
    // this wave converted is written
    wait_vm_asm<2>();
    wait_lgkmcnt<0>();
    bare_barrier();
    issue_aux(t + 6);
    if (!live) {
      issue_codes(t + 4, kres, k_codes, ks_ring);
      issue_codes(t + 3, vres, v_codes, vs_ring);
      convert_k(t + 2);
      convert_v(t + 1);
      return;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    float psum = 0.f, mx = -INFINITY;
    bf16x8 pb[2][2];
    bf16x8 kf[kWdKAhead + 1], vf[kWdVAhead + 1];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) nxt[kb][r] = 0.f;
#pragma unroll
    for (int i = 0; i < kWdKAhead; ++i) kf[i] = kfrag(t + 1, i);
    // sixteen products of S(t + 1), each with two of tile t's exponentials,
    // then sixteen of P V, each with the maxima of two of tile t + 1's logits.
    // The empty asm statements keep the running sum and maximum in their place.
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i == 1) issue_codes(t + 4, kres, k_codes, ks_ring);
      if (i == 3) issue_codes(t + 3, vres, v_codes, vs_ring);
      if (i + kWdKAhead < 16) kf[(i + kWdKAhead) % (kWdKAhead + 1)] = kfrag(t + 1, i + kWdKAhead);
      if (i >= 16 - kWdVAhead) vf[i - (16 - kWdVAhead)] = vfrag(t, i - (16 - kWdVAhead));
      nxt[i >> 3] = mfma32x32x16(kf[i % (kWdKAhead + 1)], qf[i & 7], nxt[i >> 3]);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int e = 2 * i + u, kb = e >> 4, r = e & 15;
        const float x = __builtin_amdgcn_exp2f(fmaf(cur[kb][r], scale, -m_use));
        psum += x;
        pb[kb][r >> 3][r & 7] = (bf16)x;
      }
      asm volatile("" ::"v"(psum));
      __builtin_amdgcn_sched_barrier(0);
    }
    l_part += psum;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + kWdVAhead < 16) vf[(i + kWdVAhead) % (kWdVAhead + 1)] = vfrag(t, i + kWdVAhead);
      o_acc[i & 3] = mfma32x32x16(vf[i % (kWdVAhead + 1)], pb[i >> 3][(i >> 2) & 1], o_acc[i & 3]);
      mx = fmaxf(mx, fmaxf(nxt[i >> 3][2 * (i & 7)], nxt[i >> 3][2 * (i & 7) + 1]));
      asm volatile("" ::"v"(mx));
      if (i == 2) convert_k(t + 2);
      if (i == 7) convert_v(t + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (t + 1 < t_hi) {
      if ((t + 2) * kTileK > key_end) mx = tile_max(t + 1, nxt);
      else mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
      rescale(mx);
    }
  };
  int t = t_lo;
  for (; t + 1 < t_hi; t += 2) {
    step(t, st_a, st_b);
    step(t + 1, st_b, st_a);
  }
  if (t < t_hi) step(t, st_a, st_b);
  wait_vm_asm<0>();  // every copy has landed before the workgroup's LDS is given away

  if (!live) return;
  const float l_tot = l_part + __shfl_xor(l_part, 32);
  if (q_ok) write_query(a, pair, un.split, hl, o_acc, m_run, l_tot);
}

// Combines the key splits of each (row, head): m = max_s m_s, O = sum_s
// 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s, the sums in split order.  32 lanes
// per (row, head): lane s holds splits s and 32 + s's max and sum, and each
// lane sums 4 dimensions, the O_s of four splits in flight at a time.
__global__ __launch_bounds__(256) void quant_attention_merge_kernel(const float* __restrict__ part_o,
                                                                    const float* __restrict__ part_ml, int splits,
                                                                    int64_t pairs, bf16* __restrict__ out,
                                                                    float* __restrict__ lse) {
  const int64_t pair = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (pair >= pairs) return;
  const int lane = threadIdx.x & 31;
  float2 ml[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    ml[i] = float2{-INFINITY, 0.f};
    const int s = lane + 32 * i;
    if (s < splits) ml[i] = *reinterpret_cast<const float2*>(part_ml + (s * pairs + pair) * 2);
  }
  float m = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
  for (int st = 16; st > 0; st >>= 1) m = fmaxf(m, __shfl_xor(m, st));
  float w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i].x - m);
  const float* po = part_o + pair * kDh + lane * 4;
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += 4) {
    f32x4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (s0 + i < splits) v[i] = *reinterpret_cast<const f32x4*>(po + (s0 + i) * pairs * kDh);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = s0 + i;
      const float ws = __shfl(s < 32 ? w[0] : w[1], s & 31, 32);
      l += ws * __shfl(s < 32 ? ml[0].y : ml[1].y, s & 31, 32);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += ws * v[i][j];
    }
  }
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

hipError_t launch_quant_attention(const Ragged& rg, int H, const QuantPool& p, const void* q, const int32_t* read_slots,
                                  void* out, float* lse, float* part, size_t part_bytes, hipStream_t s) {
  const int64_t rows = rg.cu_rows[rg.batch];
  if (rows == 0) return hipSuccess;
  QAttnArgs a;
  a.p = p;
  a.q = (const bf16*)q;
  a.slots = read_slots;
  a.out = (bf16*)out;
  a.lse = lse;
  a.H = H;
  a.rep = H / p.heads;
  a.rg = rg;
  const int64_t pairs = rows * H;
  int64_t tiles = 0;
  int max_kt = 0;
  for (int b = 0; b < rg.batch; ++b) {
    a.rg.tile_start[b] = (int)tiles;
    tiles += ((int64_t)(rg.cu_rows[b + 1] - rg.cu_rows[b]) * a.rep + 255) / 256;
    max_kt = std::max(max_kt, (rg.cu_keys[b + 1] - rg.cu_keys[b] + kTileK - 1) / kTileK);
  }
  a.rg.tile_start[rg.batch] = (int)tiles;
  const int64_t fit = (int64_t)(part_bytes / ((kDh + 2) * sizeof(float))) / pairs;
  int splits = (int)std::max<int64_t>(1, std::min<int64_t>({fit, kMaxSplits, (int64_t)max_kt, (512 + tiles * p.heads - 1) / (tiles * p.heads)}));
  a.splits = splits;
  a.part_o = part;
  a.part_ml = part ? part + (size_t)splits * pairs * kDh : nullptr;
  hipLaunchKernelGGL(quant_attention_wide_kernel, dim3((unsigned)(tiles * p.heads * splits)), dim3(512), 0, s, a);
  if (splits > 1)
    hipLaunchKernelGGL(quant_attention_merge_kernel, dim3((unsigned)((pairs + 7) / 8)), dim3(256), 0, s,
                       (const float*)a.part_o, (const float*)a.part_ml, splits, pairs, a.out, lse);
  return hipGetLastError();
}

}  // namespace acache
