// Internal interface between the entry points of kv.h and the gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>

// split, norm and rotation of packed rows (rope_qkv, rope_qkv_bwd, kv_append)
struct RopeParams {
  const void* qkv;   // bf16 rows of (Hq + 2 Hkv) * d, ld elements apart
  long long ld;
  const void* wq;    // bf16 [d], or null with wk: no norm
  const void* wk;
  float eps;
  const float* table;  // [npos][rot / 2][2]
  int npos, rot, interleaved;
  const int* pos;    // [T], or null (rope_qkv): position n of token b * N + n
  void* q;           // bf16 [B, Hq, N, d]; kv_append: [T, Hq, d]
  void* k;           // bf16 [B, Hkv, N, d]; kv_append: the cache
  void* v;
  int T, N, Hq, Hkv;
  // rope_qkv_bwd: q, k, v are their gradients (read)
  void* dqkv = nullptr;
  long long dld = 0;
  float* dwq = nullptr;
  float* dwk = nullptr;
  float* partial = nullptr;  // [workgroups][2][d]
  // kv_append
  const int* seq = nullptr;
  const int* pages = nullptr;
  int S = 0, W = 0, page_log2 = 0, num_pages = 0;
  float k_descale = 1.f, v_descale = 1.f;
};

int rope_qkv_launch(const RopeParams& p, int d, hipStream_t stream);
int rope_qkv_bwd_launch(const RopeParams& p, int d, hipStream_t stream);
int rope_qkv_bwd_workgroups(long long T, long long heads, int d);
int kv_append_launch(const RopeParams& p, int d, bool fp8, hipStream_t stream);

struct DecodeParams {
  const void* q;
  const void* k;
  const void* v;
  const int* pages;
  const int* lens;
  void* o;
  float* lse;
  void* ws;
  int B, Hq, Hkv, W, page_log2, num_pages;
  float scale_log2;  // scale * log2(e), times k_descale
  float out_scale;   // v_descale
};

int kv_decode_launch(const DecodeParams& p, int d, bool fp8, hipStream_t stream);
long long kv_decode_bytes(int B, int Hq, int Hkv, int d);
