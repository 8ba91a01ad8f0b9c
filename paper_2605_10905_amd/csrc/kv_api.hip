// C-ABI entry points of the rotary and paged-cache operators: argument checks, launch.  See include/kv.h.
#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kv.h"
#include "kv_kernels.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// A de-scale that 32 bits can work with: 1 / sum of up to 2^30 probabilities times it is still a normal number.
bool descale_fits(float x) { return x >= 0x1p-96f && x <= FLT_MAX; }

// what rope_qkv, its backward and kv_append have in common
int check_rows(const void* qkv, bool need_qkv, long long ld, const void* wq, const void* wk, float eps, const float* table, int npos, int rot,
               long long T, int Hq, int Hkv, int d) {
  if ((need_qkv && !qkv) || (rot > 0 && !table) || !wq != !wk) return ATTN_ERR_NULL;
  if (T <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv != 0) return ATTN_ERR_SHAPE;
  if (rot < 0 || rot > d || (rot > 0 && npos <= 0)) return ATTN_ERR_SHAPE;
  if (qkv && (ld < ((long long)Hq + 2ll * Hkv) * d || ld % 8 != 0)) return ATTN_ERR_SHAPE;
  if (misaligned(qkv, 16) || misaligned(wq, 16) || misaligned(wk, 16) || misaligned(table, 16)) return ATTN_ERR_SHAPE;
  if ((d != 64 && d != 128) || rot % 16 != 0) return ATTN_ERR_UNSUPPORTED;
  if (wq && !(eps >= 0.0f)) return ATTN_ERR_UNSUPPORTED;
  if (T > (0x7fffffffll - 1023) / ((long long)Hq + 2ll * Hkv)) return ATTN_ERR_UNSUPPORTED;  // rows are counted in 32 bits, a task past the last
  return ATTN_OK;
}

int check_pages(int W, int page_size, int num_pages) {
  if (W <= 0 || page_size <= 0 || num_pages <= 0) return ATTN_ERR_SHAPE;
  if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return ATTN_ERR_UNSUPPORTED;
  if ((long long)W * page_size > (1ll << 30)) return ATTN_ERR_UNSUPPORTED;
  return ATTN_OK;
}

RopeParams row_params(const void* qkv, long long ld, const void* wq, const void* wk, float eps, const float* table, int npos, int rot, int interleaved,
                      const int* pos, int T, int N, int Hq, int Hkv) {
  RopeParams p;
  p.qkv = qkv; p.ld = ld; p.wq = wq; p.wk = wk; p.eps = eps;
  p.table = table; p.npos = npos; p.rot = rot; p.interleaved = interleaved ? 1 : 0; p.pos = pos;
  p.q = p.k = p.v = nullptr;
  p.T = T; p.N = N; p.Hq = Hq; p.Hkv = Hkv;
  return p;
}

}  // namespace

extern "C" {

int rope_qkv(const void* qkv, long long ld, const void* q_weight, const void* k_weight, float eps, const float* table, int npos, int rot,
             int interleaved, const int* pos, void* q, void* k, void* v, int B, int Hq, int Hkv, int N, int d, void* stream) {
  if (!q || !k || !v) return ATTN_ERR_NULL;
  if (B <= 0 || N <= 0) return ATTN_ERR_SHAPE;
  const long long T = (long long)B * N;
  const int st = check_rows(qkv, true, ld, q_weight, k_weight, eps, table, npos, rot, T, Hq, Hkv, d);
  if (st != ATTN_OK) return st;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(pos, 4)) return ATTN_ERR_SHAPE;
  if (rot > 0 && !pos && N > npos) return ATTN_ERR_SHAPE;
  RopeParams p = row_params(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, (int)T, N, Hq, Hkv);
  p.q = q; p.k = k; p.v = v;
  return rope_qkv_launch(p, d, (hipStream_t)stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

int rope_qkv_bwd(const void* dq, const void* dk, const void* dv, const void* qkv, long long ld, const void* q_weight, const void* k_weight,
                 float eps, const float* table, int npos, int rot, int interleaved, const int* pos, void* dqkv, long long dld, float* dq_weight,
                 float* dk_weight, float* workspace, int B, int Hq, int Hkv, int N, int d, void* stream) {
  const bool norm = q_weight || k_weight;
  if (!dq || !dk || !dv || !dqkv || (norm && (!dq_weight || !dk_weight || !workspace))) return ATTN_ERR_NULL;
  if (B <= 0 || N <= 0) return ATTN_ERR_SHAPE;
  const long long T = (long long)B * N;
  const int st = check_rows(norm ? qkv : nullptr, norm, ld, q_weight, k_weight, eps, table, npos, rot, T, Hq, Hkv, d);
  if (st != ATTN_OK) return st;
  if (misaligned(dq, 16) || misaligned(dk, 16) || misaligned(dv, 16) || misaligned(dqkv, 16) || misaligned(pos, 4)) return ATTN_ERR_SHAPE;
  if (norm && (misaligned(dq_weight, 4) || misaligned(dk_weight, 4) || misaligned(workspace, 16))) return ATTN_ERR_SHAPE;
  if (dld < ((long long)Hq + 2ll * Hkv) * d || dld % 8 != 0) return ATTN_ERR_SHAPE;
  if (rot > 0 && !pos && N > npos) return ATTN_ERR_SHAPE;
  RopeParams p = row_params(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, (int)T, N, Hq, Hkv);
  p.q = (void*)dq; p.k = (void*)dk; p.v = (void*)dv;
  p.dqkv = dqkv; p.dld = dld;
  p.dwq = dq_weight; p.dwk = dk_weight; p.partial = workspace;
  return rope_qkv_bwd_launch(p, d, (hipStream_t)stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

long long rope_qkv_bwd_workspace_bytes(int B, int Hq, int Hkv, int N, int d) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || N <= 0 || d <= 0) return 0;
  return (long long)rope_qkv_bwd_workgroups((long long)B * N, (long long)Hq + 2ll * Hkv, d) * 2 * d * (long long)sizeof(float);
}

int kv_append(const void* qkv, long long ld, const void* q_weight, const void* k_weight, float eps, const float* table, int npos, int rot,
              int interleaved, const int* pos, const int* seq, const int* pages, void* q, void* k_cache, void* v_cache, int T, int S, int Hq,
              int Hkv, int d, int W, int page_size, int num_pages, int dtype, float k_descale, float v_descale, void* stream) {
  if (!pos || !pages || !q || !k_cache || !v_cache) return ATTN_ERR_NULL;
  if (dtype != ATTN_BF16 && dtype != ATTN_FP8_E4M3) return ATTN_ERR_DTYPE;
  int st = check_rows(qkv, true, ld, q_weight, k_weight, eps, table, npos, rot, T, Hq, Hkv, d);
  if (st != ATTN_OK) return st;
  st = check_pages(W, page_size, num_pages);
  if (st != ATTN_OK) return st;
  if (S <= 0 || (!seq && T > S)) return ATTN_ERR_SHAPE;
  if (misaligned(q, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(pos, 4) || misaligned(seq, 4) || misaligned(pages, 4))
    return ATTN_ERR_SHAPE;
  const bool fp8 = dtype == ATTN_FP8_E4M3;
  if (fp8 && (!descale_fits(k_descale) || !descale_fits(v_descale))) return ATTN_ERR_UNSUPPORTED;
  RopeParams p = row_params(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, T, 0, Hq, Hkv);
  p.q = q; p.k = k_cache; p.v = v_cache;
  p.seq = seq; p.pages = pages;
  p.S = S; p.W = W; p.page_log2 = __builtin_ctz((unsigned)page_size); p.num_pages = num_pages;
  p.k_descale = k_descale; p.v_descale = v_descale;
  return kv_append_launch(p, d, fp8, (hipStream_t)stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

int kv_decode(const void* q, const void* k_cache, const void* v_cache, const int* pages, const int* lens, void* o, float* lse, void* workspace,
              int B, int Hq, int Hkv, int d, int W, int page_size, int num_pages, float scale, int dtype, float k_descale, float v_descale,
              void* stream) {
  if (!q || !k_cache || !v_cache || !pages || !lens || !o || !lse || !workspace) return ATTN_ERR_NULL;
  if (dtype != ATTN_BF16 && dtype != ATTN_FP8_E4M3) return ATTN_ERR_DTYPE;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv != 0) return ATTN_ERR_SHAPE;
  const int st = check_pages(W, page_size, num_pages);
  if (st != ATTN_OK) return st;
  if (misaligned(q, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(o, 16) || misaligned(workspace, 16) ||
      misaligned(lse, 4) || misaligned(pages, 4) || misaligned(lens, 4))
    return ATTN_ERR_SHAPE;
  if (d != 64 && d != 128) return ATTN_ERR_UNSUPPORTED;
  const bool fp8 = dtype == ATTN_FP8_E4M3;
  if (!(scale > 0.0f) || (fp8 && (!descale_fits(k_descale) || !descale_fits(v_descale)))) return ATTN_ERR_UNSUPPORTED;
  // what the scores are multiplied by: as zero or infinity it would make NaN of a hidden key's -inf, or of the largest score's 0
  const float scale_log2 = scale * kLog2e * (fp8 ? k_descale : 1.0f);
  if (!(scale_log2 >= FLT_MIN && scale_log2 <= FLT_MAX)) return ATTN_ERR_UNSUPPORTED;
  if ((long long)B * Hq > 0x00ffffffll) return ATTN_ERR_UNSUPPORTED;  // one workgroup per row has to fit a launch
  DecodeParams p;
  p.q = q; p.k = k_cache; p.v = v_cache; p.pages = pages; p.lens = lens; p.o = o; p.lse = lse; p.ws = workspace;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.W = W; p.page_log2 = __builtin_ctz((unsigned)page_size); p.num_pages = num_pages;
  p.scale_log2 = scale_log2;
  p.out_scale = fp8 ? v_descale : 1.0f;
  return kv_decode_launch(p, d, fp8, (hipStream_t)stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

long long kv_decode_workspace_bytes(int B, int Hq, int Hkv, int d) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv != 0) return 0;
  return kv_decode_bytes(B, Hq, Hkv, d);
}

}  // extern "C"
