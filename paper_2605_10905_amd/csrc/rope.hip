// Split, per-head RMS norm and rotation of a packed q|k|v projection (rope_qkv), its gradients (rope_qkv_bwd), and the same
// into a paged cache (kv_append).
//
// One pass over the rows, bound by memory: a row of d features is read once, everything between is 32-bit arithmetic in
// registers, and it is rounded once when it is written.  d / 16 lanes hold a row, each two 16-byte chunks a and b, chosen so
// that every pair of rotated features lies in one lane: chunk c of the first rot / 16 and chunk c + rot / 16, whose features
// are each other's partners when the pairs are (f, f + rot / 2); adjacent pairs lie inside a chunk anyhow.  What is not
// rotated is dealt to the remaining lanes the same way.  The mean of squares is a sum over d / 16 neighbouring lanes (quad
// permutations and a half-row mirror, no LDS).
//
// Measured, where a 1 GiB device copy runs at 5.16 TB/s: rope_qkv of 16384 tokens, 64/8 heads, d = 128 128 - 131 us (5.1 - 5.3 TB/s); kv_append of
// 9951 tokens, 32/8 heads into an e4m3 cache 45 us (5.0); rope_qkv_bwd of 8192 tokens, 16/16 heads 54 us (5.0) and 5 for the sums of the
// weights' gradients; one token 3.9 - 4.6, which is a launch.
#include "attn_device.h"
#include "kv_kernels.h"

namespace {

constexpr int kWaves = 4;
constexpr int kMostWorkgroups = 1 << 20;  // (a launch holds 2^32 threads)

constexpr int kMostPartials = 1024;  // workgroups of a backward pass, each with its sums of the weights' gradients
typedef __attribute__((ext_vector_type(4))) float f32x4;

// A wave takes kRowSpan (kv_append: kGroupSpan) steps, unless all steps can be taken by one wave each that start at once (4 waves on each of 1024
// SIMDs): the smallest calls last as long as one wave's chain (64 tokens of 64/8 heads appended by spans of 4 5.8 us, of 1 4.8).  us at span
// 1 / 3 / 4 / 6 / 8: rope_qkv of 16384 tokens of 64/8 heads, d = 128 157 / 130 / 128 / 132 / 131, of 30000 of 8/1 - / 40.6 / 41.0 / 42.6 / 47.3, of
// 1000 of 32/8 7.7 / 6.9 / 7.3 / 8.0 / 9.4; 9951 tokens of 32/8 heads into an e4m3 cache 57.6 / 45.3 / 45.0 / - / 47.9.
constexpr int kRowSpan = 3, kGroupSpan = 4, kFewTasks = 4096;

// sum over the LPR (4 or 8) neighbouring lanes of a row, the same value in all of them
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, true));   // quad_perm 1,0,3,2
  x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, true));   // quad_perm 2,3,0,1
  if constexpr (LPR == 8) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, true));  // row_half_mirror
  return x;
}

__device__ __forceinline__ void unpack(const u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(x[i] << 16);
    f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
  return u32x4{attn_pack_bf16(f[0], f[1]), attn_pack_bf16(f[2], f[3]), attn_pack_bf16(f[4], f[5]), attn_pack_bf16(f[6], f[7])};
}

// which two chunks lane j of a row holds, and whether they are rotated
struct Chunks {
  int a, b;
  bool rotated;
};
template <int LPR>
__device__ __forceinline__ Chunks chunks_of(int j, int rot) {
  const int r = rot >> 4;
  Chunks c;
  c.rotated = j < r;
  c.a = j < r ? j : r + j;
  c.b = j < r ? j + r : LPR + j;
  return c;
}

// cosine and sine of the lane's eight pairs at position `pos` (inside the table); zeros, which nobody uses, where nothing is rotated
__device__ __forceinline__ void load_angles(const RopeParams& p, const Chunks& c, int pos, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = sn[i] = 0.f;
  if (!c.rotated) return;
  const f32x4* const row = (const f32x4*)(p.table + (size_t)pos * p.rot);
  const int at0 = p.interleaved ? 2 * c.a : 4 * c.a, at1 = p.interleaved ? 2 * c.b : 4 * c.a + 2;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 t = row[(i < 2 ? at0 : at1) + (i & 1)];
    cs[2 * i] = t[0];
    sn[2 * i] = t[1];
    cs[2 * i + 1] = t[2];
    sn[2 * i + 1] = t[3];
  }
}

// The rotation (SIGN 1) or its transpose (-1) of a pair.  Pairs that are not rotated keep their features (by an angle of zero an infinity in one
// would make the other, which only shares the lane with it, NaN).  Here and in the norm the fused products are written out, so that rope_qkv and
// kv_append give the same bits.
template <int SIGN>
__device__ __forceinline__ void turn(bool rotated, float& x, float& y, float cs, float sn) {
  const float s = SIGN * sn, u = fmaf(x, cs, -(y * s)), w = fmaf(y, cs, x * s);
  x = rotated ? u : x;
  y = rotated ? w : y;
}
template <int SIGN>
__device__ __forceinline__ void rotate(bool rotated, bool interleaved, float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
  if (!interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn<SIGN>(rotated, a[i], b[i], cs[i], sn[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn<SIGN>(rotated, a[2 * i], a[2 * i + 1], cs[i], sn[i]);
      turn<SIGN>(rotated, b[2 * i], b[2 * i + 1], cs[4 + i], sn[4 + i]);
    }
  }
}

template <int LPR>
__device__ __forceinline__ float inverse_rms(const float (&a)[8], const float (&b)[8], float eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(a[i], a[i], fmaf(b[i], b[i], s));
  // 1 / sqrt, not the approximate reciprocal root: a row's error would be common to all of its features
  return 1.f / sqrtf(fmaf(row_sum<LPR>(s), 1.f / (16 * LPR), eps));
}

// eight codes of x / descale, round to nearest even, saturated; NaN stays NaN
__device__ __forceinline__ u32x2 to_e4m3(const float (&x)[8], float descale) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = x[i] / descale;
    y[i] = y[i] > 448.f ? 448.f : y[i] < -448.f ? -448.f : y[i];
  }
  int w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], w[i], false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w[i], true);
  }
  return u32x2{(uint32_t)w[0], (uint32_t)w[1]};
}

// norm and rotation of a row of q or k; NaN where its position is not in the table
template <int LPR>
__device__ __forceinline__ void turn_row(const RopeParams& p, const Chunks& c, float (&a)[8], float (&b)[8], const u32x4 (&weight)[2], const float (&cs)[8], const float (&sn)[8], bool good) {
  if (p.wq) {
    float wa[8], wb[8];
    unpack(weight[0], wa);
    unpack(weight[1], wb);
    const float r = inverse_rms<LPR>(a, b, p.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a[i] = a[i] * r * wa[i];
      b[i] = b[i] * r * wb[i];
    }
  }
  rotate<1>(c.rotated, p.interleaved, a, b, cs, sn);
  if (!good) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = b[i] = __builtin_nanf("");
  }
}
__device__ __forceinline__ void load_weights(const RopeParams& p, const Chunks& c, u32x4 (&wq)[2], u32x4 (&wk)[2]) {
  if (!p.wq) return;
  wq[0] = *(const u32x4*)((const char*)p.wq + c.a * 16);
  wq[1] = *(const u32x4*)((const char*)p.wq + c.b * 16);
  wk[0] = *(const u32x4*)((const char*)p.wk + c.a * 16);
  wk[1] = *(const u32x4*)((const char*)p.wk + c.b * 16);
}

// A lane's row: head h of token t.  rope_qkv and its backward deal the rows of all tokens to the waves one after the other, 64 / (d / 16) at a
// time, so that no lane idles whatever the number of heads is (a wave for each token / this, us: 30000 tokens of 8/1 heads 47.4 / 40.5, backward
// 68.2 / 53.5; 32768 of 16/4, d = 64 51.9 / 47.2, backward 79 / 67; 16384 of 64/8 128.7 / 129.9).
struct Place {
  int t, h;
};
// (ONE: all rows that a wave holds at once are of one token, a multiple of them its heads; positions then come by scalar loads: backward of 16384
// tokens of 32/8 heads 121 -> 117 us.)
template <bool ONE>
__device__ __forceinline__ Place place_of(int row, int H) {
  Place x;
  x.t = (ONE ? __builtin_amdgcn_readfirstlane(row) : row) / H;
  x.h = row - x.t * H;
  return x;
}
// scalar load of what no kernel writes while this one runs
__device__ __forceinline__ int scalar_load(const int* p, size_t i) { return ((const __attribute__((address_space(4))) int*)p)[i]; }

// One task of rope_qkv, by one wave: `span` times 64 / (d / 16) consecutive rows.  A token's angles are fetched where a lane's row is the first of
// it, the rows and positions one step ahead.
template <int D>
__device__ __forceinline__ void rope_task(const RopeParams& p, int rows, int span, int task) {
  constexpr int LPR = D / 16, RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, H = p.Hq + 2 * p.Hkv;
  const Chunks c = chunks_of<LPR>(lane % LPR, p.rot);
  const int first = task * span * RPW + lane / LPR, steps = min(span, (rows - task * span * RPW + RPW - 1) / RPW);

  u32x4 xa, xb, wq[2], wk[2];
  int pos = 0;
  auto fetch = [&](const Place& x, bool other) __attribute__((always_inline)) {  // (of another token; rows past the last re-read it)
    const int t = min(x.t, p.T - 1), h = x.t < p.T ? x.h : H - 1;
    if (other && p.pos) pos = p.pos[t];
    const char* const src = (const char*)p.qkv + ((size_t)t * p.ld + (size_t)h * D) * 2;
    xa = *(const u32x4*)(src + c.a * 16);
    xb = *(const u32x4*)(src + c.b * 16);
  };
  Place next = place_of<false>(min(first, rows - 1), H);
  if (first >= rows) next.t = p.T;
  fetch(next, true);
  load_weights(p, c, wq, wk);
  const int whole = RPW / H, rest = RPW - whole * H;  // tokens and heads that RPW rows are

  int have = -1, bb = 0, n = 0;  // the token that the following are of
  bool good = false;
  float cs[8], sn[8];
  for (int g = 0; g < steps; ++g) {
    const Place x = next;
    const u32x4 ya = xa, yb = xb;
    if (x.t != have) {
      have = x.t;
      bb = x.t / p.N;
      n = x.t - bb * p.N;
      const int at = p.pos ? pos : n;
      good = p.rot == 0 || (unsigned)at < (unsigned)p.npos;
      load_angles(p, c, good ? at : 0, cs, sn);
    }
    next.h += rest;
    next.t += whole;
    if (next.h >= H) {
      next.h -= H;
      ++next.t;
    }
    if (g + 1 < steps) fetch(next, next.t != x.t);
    if (x.t >= p.T) continue;
    const bool is_q = x.h < p.Hq, is_v = x.h >= p.Hq + p.Hkv;
    float a[8], b[8];
    unpack(ya, a);
    unpack(yb, b);
    if (!is_v) turn_row<LPR>(p, c, a, b, is_q ? wq : wk, cs, sn, good);
    const int hk = is_q ? x.h : is_v ? x.h - p.Hq - p.Hkv : x.h - p.Hq, Hk = is_q ? p.Hq : p.Hkv;
    char* const dst = (char*)(is_q ? p.q : is_v ? p.v : p.k) + (((size_t)bb * Hk + hk) * p.N + n) * (D * 2);
    *(u32x4*)(dst + c.a * 16) = is_v ? ya : pack(a);
    *(u32x4*)(dst + c.b * 16) = is_v ? yb : pack(b);
  }
}

// One task of kv_append, by one wave: `span` groups of 64 / (d / 16) consecutive heads of one token.  The token's position, page and angles and the
// norms' weights are fetched once for all of them, the rows of the next group while the ones of this group are computed.  (Rows dealt as
// rope_qkv's: 9951 tokens of 32/8 heads into an e4m3 cache 45.4 -> 47 - 49 us, 28/4 41 -> 43 - 47.)
template <int D, bool FP8>
__device__ __forceinline__ void append_task(const RopeParams& p, int groups, int span, int task) {
  constexpr int LPR = D / 16, RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, j = lane % LPR, H = p.Hq + 2 * p.Hkv;
  const int spans = (groups + span - 1) / span, t = task / spans, g0 = (task - t * spans) * span, g1 = min(g0 + span, groups);
  const Chunks c = chunks_of<LPR>(j, p.rot);

  const char* const row = (const char*)p.qkv + (size_t)t * p.ld * 2;
  auto fetch = [&](int g, u32x4& xa, u32x4& xb) __attribute__((always_inline)) {
    const char* const src = row + (size_t)min(g * RPW + lane / LPR, H - 1) * (D * 2);  // (heads past the last are not written)
    xa = *(const u32x4*)(src + c.a * 16);
    xb = *(const u32x4*)(src + c.b * 16);
  };
  u32x4 xa, xb, wq[2], wk[2];
  fetch(g0, xa, xb);
  load_weights(p, c, wq, wk);

  const int pos = scalar_load(p.pos, t);
  if (pos < 0) return;  // padding
  const int seq = p.seq ? scalar_load(p.seq, t) : t;
  const bool good = (p.rot == 0 || pos < p.npos) && (unsigned)seq < (unsigned)p.S;
  int entry = -1;
  if (good && (pos >> p.page_log2) < p.W) entry = scalar_load(p.pages, (size_t)seq * p.W + (pos >> p.page_log2));
  if ((unsigned)entry >= (unsigned)p.num_pages) entry = -1;
  float cs[8], sn[8];
  load_angles(p, c, good ? pos : 0, cs, sn);

  for (int g = g0; g < g1; ++g) {
    const u32x4 ya = xa, yb = xb;
    if (g + 1 < g1) fetch(g + 1, xa, xb);
    const int h = g * RPW + lane / LPR;
    if (h >= H) continue;
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
    float a[8], b[8];
    unpack(ya, a);
    unpack(yb, b);
    if (!is_v) turn_row<LPR>(p, c, a, b, is_q ? wq : wk, cs, sn, good);
    char* dst = (char*)p.q + ((size_t)t * p.Hq + h) * (D * 2);
    if (!is_q) {
      if (!good || entry < 0) continue;
      const int hk = is_v ? h - p.Hq - p.Hkv : h - p.Hq;
      const size_t place = (((size_t)entry * p.Hkv + hk) << p.page_log2) + (pos & ((1 << p.page_log2) - 1));
      dst = (char*)(is_v ? p.v : p.k) + place * (D * (FP8 ? 1 : 2));
      if constexpr (FP8) {
        const float descale = is_v ? p.v_descale : p.k_descale;
        *(u32x2*)(dst + c.a * 8) = to_e4m3(a, descale);
        *(u32x2*)(dst + c.b * 8) = to_e4m3(b, descale);
        continue;
      }
    }
    *(u32x4*)(dst + c.a * 16) = is_v ? ya : pack(a);
    *(u32x4*)(dst + c.b * 16) = is_v ? yb : pack(b);
  }
}

template <int D>
__global__ void __launch_bounds__(kWaves * 64) rope_qkv_kernel(const RopeParams p, int rows, int span, int tasks) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int task = blockIdx.x * kWaves + w; task < tasks; task += gridDim.x * kWaves) rope_task<D>(p, rows, span, task);
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kWaves * 64) kv_append_kernel(const RopeParams p, int groups, int span, int tasks) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int task = blockIdx.x * kWaves + w; task < tasks; task += gridDim.x * kWaves) append_task<D, FP8>(p, groups, span, task);
}

// The gradients.  A workgroup walks tasks (64 / (d / 16) consecutive rows) a grid apart and keeps what its lanes add to the
// weights' gradients in registers; the sums over lanes, waves and workgroups follow in a fixed order.
template <int D, bool NORM, bool ONE>
__global__ void __launch_bounds__(kWaves * 64) rope_qkv_bwd_kernel(const RopeParams p, int rows, int tasks) {
  constexpr int LPR = D / 16, RPW = 64 / LPR;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int j = lane % LPR, H = p.Hq + 2 * p.Hkv;
  const Chunks c = chunks_of<LPR>(j, p.rot);
  float acc[2][2][8];  // [q, k][chunk a, b]
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[0][0][i] = acc[0][1][i] = acc[1][0][i] = acc[1][1][i] = 0.f;

  for (int task = blockIdx.x * kWaves + w; task < tasks; task += gridDim.x * kWaves) {
    const int row = task * RPW + lane / LPR;
    if (row >= rows) continue;
    const Place x = place_of<ONE>(row, H);
    const int t = x.t, h = x.h;
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
    const int hk = is_q ? h : is_v ? h - p.Hq - p.Hkv : h - p.Hq, Hk = is_q ? p.Hq : p.Hkv;
    const int n = t % p.N, bb = t / p.N;
    const char* const src = (const char*)(is_q ? p.q : is_v ? p.v : p.k) + (((size_t)bb * Hk + hk) * p.N + n) * (D * 2);
    char* const dst = (char*)p.dqkv + ((size_t)t * p.dld + (size_t)h * D) * 2;
    const u32x4 ga4 = *(const u32x4*)(src + c.a * 16), gb4 = *(const u32x4*)(src + c.b * 16);
    if (is_v) {
      *(u32x4*)(dst + c.a * 16) = ga4;
      *(u32x4*)(dst + c.b * 16) = gb4;
      continue;
    }
    const int pos = !p.pos ? n : ONE ? scalar_load(p.pos, t) : p.pos[t];
    const bool good = p.rot == 0 || (unsigned)pos < (unsigned)p.npos;
    float a[8], b[8], cs[8], sn[8];
    unpack(ga4, a);
    unpack(gb4, b);
    load_angles(p, c, good ? pos : 0, cs, sn);
    rotate<-1>(c.rotated, p.interleaved, a, b, cs, sn);
    if (!good) {
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = b[i] = __builtin_nanf("");
    }
    if constexpr (NORM) {
      const char* const xsrc = (const char*)p.qkv + ((size_t)t * p.ld + (size_t)h * D) * 2;
      const char* const wsrc = (const char*)(is_q ? p.wq : p.wk);
      float xa[8], xb[8], wa[8], wb[8];
      unpack(*(const u32x4*)(xsrc + c.a * 16), xa);
      unpack(*(const u32x4*)(xsrc + c.b * 16), xb);
      unpack(*(const u32x4*)(wsrc + c.a * 16), wa);
      unpack(*(const u32x4*)(wsrc + c.b * 16), wb);
      const float r = inverse_rms<LPR>(xa, xb, p.eps);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xa[i] *= r;
        xb[i] *= r;
        const float da = a[i] * xa[i], db = b[i] * xb[i];
        acc[0][0][i] += is_q ? da : 0.f;
        acc[0][1][i] += is_q ? db : 0.f;
        acc[1][0][i] += is_q ? 0.f : da;
        acc[1][1][i] += is_q ? 0.f : db;
        a[i] *= wa[i];
        b[i] *= wb[i];
        dot += a[i] * xa[i] + b[i] * xb[i];
      }
      dot = row_sum<LPR>(dot) * (1.f / D);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = r * (a[i] - xa[i] * dot);
        b[i] = r * (b[i] - xb[i] * dot);
      }
    }
    *(u32x4*)(dst + c.a * 16) = pack(a);
    *(u32x4*)(dst + c.b * 16) = pack(b);
  }

  if constexpr (NORM) {
    // over the rows that the lanes held (those that agree mod LPR) and the waves, through LDS: a column is the sum of 64 / LPR * kWaves
    // values, taken by two (d = 64) or one of the threads.  (By exchanges between lanes: 128 of them at d = 64, 2 us.)
    constexpr int PITCH = 2 * D + 4;  // floats of a row of sums: q's d, k's d
    __shared__ __attribute__((aligned(16))) float part[kWaves * RPW][PITCH];
    float* const mine = part[w * RPW + lane / LPR];
#pragma unroll
    for (int qk = 0; qk < 2; ++qk)
#pragma unroll
      for (int ab = 0; ab < 2; ++ab)
#pragma unroll
        for (int i = 0; i < 8; i += 4)
          *(f32x4*)(mine + qk * D + (ab ? c.b : c.a) * 8 + i) = f32x4{acc[qk][ab][i], acc[qk][ab][i + 1], acc[qk][ab][i + 2], acc[qk][ab][i + 3]};
    __syncthreads();
    constexpr int SHARE = kWaves * 64 / (2 * D);  // threads of a column
    const int col = threadIdx.x % (2 * D), at = threadIdx.x / (2 * D);
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves * RPW / SHARE; ++i) x += part[i * SHARE + at][col];
    if constexpr (SHARE == 2) {
      __syncthreads();
      part[at][col] = x;
      __syncthreads();
      x = part[0][col] + part[1][col];
    }
    if (at == 0) p.partial[(size_t)blockIdx.x * (2 * D) + col] = x;
  }
}

// the sums over workgroups: one workgroup for 16 of the 2 d columns; four threads take their four columns of a row each, so that at most
// four loads of every thread are under way at once
template <int D>
__global__ void __launch_bounds__(1024) rope_weight_sum_kernel(const float* partial, int workgroups, float* dwq, float* dwk) {
  __shared__ f32x4 part[16][4];
  const int c4 = threadIdx.x & 3, at = threadIdx.x >> 2, w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float* const src = partial + blockIdx.x * 16 + c4 * 4;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kMostPartials / 256; ++i)
    if (i * 256 + at < workgroups) x += *(const f32x4*)(src + (size_t)(i * 256 + at) * (2 * D));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int m = 4; m < 64; m *= 2) x[i] += __shfl_xor(x[i], m);
  }
  if (lane < 4) part[w][lane] = x;
  __syncthreads();
  if (threadIdx.x < 16) {
    const int col = blockIdx.x * 16 + threadIdx.x;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) y += part[i][threadIdx.x >> 2][threadIdx.x & 3];
    (col < D ? dwq : dwk)[col % D] = y;
  }
}

int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

// Rows of all tokens (below 2^31), and the tasks of `span` times 64 / (d / 16) of them.
int rows_of(const RopeParams& p) { return p.T * (p.Hq + 2 * p.Hkv); }
int tasks_of(int rows, int d, int span) { return (int)(((long long)rows + span * (1024 / d) - 1) / (span * (1024 / d))); }

}  // namespace

int rope_qkv_launch(const RopeParams& p, int d, hipStream_t stream) {
  const int rows = rows_of(p), span = tasks_of(rows, d, 1) <= kFewTasks ? 1 : kRowSpan, tasks = tasks_of(rows, d, span);
  const int grid = min((tasks - 1) / kWaves + 1, kMostWorkgroups);
  if (d == 128) rope_qkv_kernel<128><<<grid, kWaves * 64, 0, stream>>>(p, rows, span, tasks);
  else rope_qkv_kernel<64><<<grid, kWaves * 64, 0, stream>>>(p, rows, span, tasks);
  return launched();
}

int kv_append_launch(const RopeParams& p, int d, bool fp8, hipStream_t stream) {
  const int groups = tasks_of(p.Hq + 2 * p.Hkv, d, 1), span = (long long)p.T * groups <= kFewTasks ? 1 : kGroupSpan;
  const int tasks = p.T * ((groups + span - 1) / span), grid = min((tasks - 1) / kWaves + 1, kMostWorkgroups);
  if (d == 128 && fp8) kv_append_kernel<128, true><<<grid, kWaves * 64, 0, stream>>>(p, groups, span, tasks);
  else if (d == 128) kv_append_kernel<128, false><<<grid, kWaves * 64, 0, stream>>>(p, groups, span, tasks);
  else if (fp8) kv_append_kernel<64, true><<<grid, kWaves * 64, 0, stream>>>(p, groups, span, tasks);
  else kv_append_kernel<64, false><<<grid, kWaves * 64, 0, stream>>>(p, groups, span, tasks);
  return launched();
}

int rope_qkv_bwd_workgroups(long long T, long long heads, int d) {
  constexpr long long kEnough = kMostPartials * kWaves * (1024 / 64);  // tokens or heads that take every workgroup (so that any product fits)
  const long long rows = (T < kEnough ? T : kEnough) * (heads < kEnough ? heads : kEnough);
  const long long per = d >= 1024 ? 1 : 1024 / d, tasks = (rows + per - 1) / per, wgs = (tasks + kWaves - 1) / kWaves;
  return (int)(wgs < kMostPartials ? wgs : kMostPartials);
}

namespace {

template <int D, bool ONE>
int launch_bwd(const RopeParams& p, hipStream_t stream) {
  const int rows = rows_of(p), tasks = tasks_of(rows, D, 1), grid = rope_qkv_bwd_workgroups(p.T, p.Hq + 2 * p.Hkv, D);
  if (!p.wq) {
    rope_qkv_bwd_kernel<D, false, ONE><<<grid, kWaves * 64, 0, stream>>>(p, rows, tasks);
    return launched();
  }
  rope_qkv_bwd_kernel<D, true, ONE><<<grid, kWaves * 64, 0, stream>>>(p, rows, tasks);
  if (launched() != 0) return 1;
  rope_weight_sum_kernel<D><<<2 * D / 16, 1024, 0, stream>>>(p.partial, grid, p.dwq, p.dwk);
  return launched();
}

}  // namespace

int rope_qkv_bwd_launch(const RopeParams& p, int d, hipStream_t stream) {
  if ((p.Hq + 2 * p.Hkv) % (1024 / d) == 0) return d == 128 ? launch_bwd<128, true>(p, stream) : launch_bwd<64, true>(p, stream);
  return d == 128 ? launch_bwd<128, false>(p, stream) : launch_bwd<64, false>(p, stream);
}
