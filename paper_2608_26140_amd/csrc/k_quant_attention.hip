// Read-slot attention over the 8-bit KV cache (gfx950).
#include "internal.h"
#include "quant.h"

namespace acache {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

constexpr int kDh = 128;

struct QAttnArgs {
  QuantPool p;
  const bf16* q;
  const int32_t* slots;
  bf16* out;
  float* lse;
  int H;
  Ragged rg;
};

// One wavefront per (row, head): eight lanes a key, 16 dimensions each.
__global__ __launch_bounds__(64) void quant_attention_row_kernel(QAttnArgs a) {
  const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, part = lane & 7, kg = lane >> 3;
  int b = 0;
  while (a.rg.cu_rows[b + 1] <= row) ++b;
  const int g = h / (a.H / a.p.heads);
  const int k0 = a.rg.cu_keys[b], S = a.rg.cu_keys[b + 1] - k0;
  const float scale = kLog2e * rsqrtf((float)kDh);
  const bf16* qp = a.q + ((int64_t)row * a.H + h) * kDh + part * 16;
  float q[16], o[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    q[j] = (float)qp[j] * scale;
    o[j] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int j0 = 0; j0 < S; j0 += 8) {
    const int j = j0 + kg;
    const int s = j < S ? a.slots[k0 + j] : -1;
    float kv[2][16];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float sc = 0.f;
      u32x4 c = {0u, 0u, 0u, 0u};
      if (s >= 0 && s < a.p.n_slots) {
        sc = a.p.scales[w][(int64_t)(s >> a.p.shift) * a.p.heads + g];
        sc = __uint_as_float(__float_as_uint(sc) & 0x7F800000u);
        if (sc > 0.f) c = *reinterpret_cast<const u32x4*>((const uint8_t*)a.p.codes[w] + (int64_t)s * a.p.ld + g * kDh + part * 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float d[4];
        decode4(c[i], d);
#pragma unroll
        for (int u = 0; u < 4; ++u) kv[w][4 * i + u] = d[u] * sc;
      }
    }
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x += q[i] * kv[0][i];
    x += __shfl_xor(x, 1);
    x += __shfl_xor(x, 2);
    x += __shfl_xor(x, 4);
    if (j < S) {
      const float mn = fmaxf(m, x);
      const float f = m == -INFINITY ? 0.f : exp2f(m - mn), e = exp2f(x - mn);
      l = l * f + e;
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] = o[i] * f + e * kv[1][i];
      m = mn;
    }
  }
#pragma unroll
  for (int st = 8; st < 64; st <<= 1) {
    const float m2 = __shfl_xor(m, st), l2 = __shfl_xor(l, st), mn = fmaxf(m, m2);
    const float f = m == -INFINITY ? 0.f : exp2f(m - mn), f2 = m2 == -INFINITY ? 0.f : exp2f(m2 - mn);
    l = l * f + l2 * f2;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = o[i] * f + __shfl_xor(o[i], st) * f2;
    m = mn;
  }
  if (kg != 0) return;
  bf16* op = a.out + ((int64_t)row * a.H + h) * kDh + part * 16;
#pragma unroll
  for (int j = 0; j < 16; ++j) op[j] = (bf16)(o[j] / l);
  if (a.lse && part == 0) a.lse[(int64_t)row * a.H + h] = (m + log2f(l)) * kLn2;
}

}  // namespace

hipError_t launch_quant_attention(const Ragged& rg, int H, const QuantPool& p, const void* q, const int32_t* read_slots,
                                  void* out, float* lse, float* part, size_t part_bytes, hipStream_t s) {
  const int rows = rg.cu_rows[rg.batch];
  if (rows == 0) return hipSuccess;
  QAttnArgs a;
  a.p = p;
  a.q = (const bf16*)q;
  a.slots = read_slots;
  a.out = (bf16*)out;
  a.lse = lse;
  a.H = H;
  a.rg = rg;
  hipLaunchKernelGGL(quant_attention_row_kernel, dim3(rows, H), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace acache
