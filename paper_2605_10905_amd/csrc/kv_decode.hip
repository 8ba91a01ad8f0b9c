// Attention of one new token per sequence over the paged cache (kv_decode).
#include "attn_device.h"
#include "kv_kernels.h"

namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ float element(const char* row, int i, bool fp8) {
  if (!fp8) return __uint_as_float((uint32_t)((const uint16_t*)row)[i] << 16);
  return __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t*)row)[i], 0);
}

// One workgroup per query row; its waves take the keys in turn, lane i the features i and i + 64.
template <int D, bool FP8>
__global__ void __launch_bounds__(kWaves * 64) kv_decode_kernel(const DecodeParams p) {
  constexpr int E = D / 64;
  __shared__ float so[kWaves][D], sm[kWaves], sl[kWaves];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int b = blockIdx.x / p.Hq, hq = blockIdx.x % p.Hq, hk = hq / (p.Hq / p.Hkv);
  const int len = min(max(p.lens[b], 0), p.W << p.page_log2);
  const uint16_t* const qrow = (const uint16_t*)p.q + (size_t)blockIdx.x * D;
  float q[E], o[E], m = -__builtin_inff(), l = 0.f;
  for (int e = 0; e < E; ++e) {
    q[e] = __uint_as_float((uint32_t)qrow[lane + 64 * e] << 16);
    o[e] = 0.f;
  }
  for (int j = w; j < len; j += kWaves) {
    const int entry = p.pages[(size_t)b * p.W + (j >> p.page_log2)];
    if ((unsigned)entry >= (unsigned)p.num_pages) continue;
    const size_t row = ((((size_t)entry * p.Hkv + hk) << p.page_log2) + (j & ((1 << p.page_log2) - 1))) * (D * (FP8 ? 1 : 2));
    float s = 0.f;
    for (int e = 0; e < E; ++e) s += q[e] * element((const char*)p.k + row, lane + 64 * e, FP8);
    for (int x = 1; x < 64; x *= 2) s += __shfl_xor(s, x);
    const float m_new = fmaxf(m, s), ref = m_new == -__builtin_inff() ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f((m - ref) * p.scale_log2), pr = __builtin_amdgcn_exp2f((s - ref) * p.scale_log2);
    for (int e = 0; e < E; ++e) o[e] = o[e] * alpha + pr * element((const char*)p.v + row, lane + 64 * e, FP8);
    l = l * alpha + pr;
    m = m_new;
  }
  for (int e = 0; e < E; ++e) so[w][lane + 64 * e] = o[e];
  if (lane == 0) {
    sm[w] = m;
    sl[w] = l;
  }
  __syncthreads();
  if (w != 0) return;
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const float ref = m == -__builtin_inff() ? 0.f : m;
  l = 0.f;
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int k = 0; k < kWaves; ++k) {
    const float a = __builtin_amdgcn_exp2f((sm[k] - ref) * p.scale_log2);
    l += sl[k] * a;
    for (int e = 0; e < E; ++e) o[e] += so[k][lane + 64 * e] * a;
  }
  const float inv = l == 0.f ? 0.f : p.out_scale / l;
  for (int e = 0; e < E; ++e) ((__bf16*)p.o)[(size_t)blockIdx.x * D + lane + 64 * e] = (__bf16)(o[e] * inv);
  if (lane == 0) p.lse[blockIdx.x] = l == 0.f ? -__builtin_inff() : (m * p.scale_log2 + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

}  // namespace

int kv_decode_launch(const DecodeParams& p, int d, bool fp8, hipStream_t stream) {
  const int grid = p.B * p.Hq;
  if (d == 128 && fp8) kv_decode_kernel<128, true><<<grid, kWaves * 64, 0, stream>>>(p);
  else if (d == 128) kv_decode_kernel<128, false><<<grid, kWaves * 64, 0, stream>>>(p);
  else if (fp8) kv_decode_kernel<64, true><<<grid, kWaves * 64, 0, stream>>>(p);
  else kv_decode_kernel<64, false><<<grid, kWaves * 64, 0, stream>>>(p);
  return hipGetLastError() == hipSuccess ? 0 : 1;
}

long long kv_decode_bytes(int, int, int, int) { return 16; }
