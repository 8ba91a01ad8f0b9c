/*
 * C ABI of libkv_mi355x.so (MI355X, gfx950): what stands around attention in a transformer layer.
 *
 *   rope_qkv, rope_qkv_bwd   between the q|k|v projection (gemm.h) and attention (attn.h): the rows of the packed
 *                            projection are split into heads, q and k are RMS-normalised per head and rotated by
 *                            their position, and q, k, v are written in attn_fwd's layout; and the gradients
 *   kv_append                the same for new tokens while generating: k and v go into a paged cache
 *   kv_decode                attention of one new token per sequence over that cache
 *
 * For a row x of d features of a query or key head at position p:
 *
 *     y = x / sqrt(mean(x^2) + eps) * weight            (without weights: y = x)
 *     z = R(p) y                                        the pair of features (i, j) is turned by the angle whose
 *                                                       cosine and sine the table holds for p and that pair:
 *       z_i = y_i cos - y_j sin,  z_j = y_j cos + y_i sin
 *
 * Only the first `rot` features are rotated.  With `interleaved` 0 pair f is (f, f + rot / 2), otherwise
 * (2 f, 2 f + 1).  Rows of v are copied.  Everything is computed in 32 bits from the stored inputs and rounded once,
 * to the type it is stored in.
 *
 * The table is float32 [npos][rot / 2][2]: cosine and sine of position p and pair f, as the caller's model defines them
 * (angle p * base^(-2 f / rot), taken in 64 bits: 32 lose the angles of far positions; or any scaled form of it).
 *
 * All pointers are DEVICE pointers.  The caller owns all buffers and keeps them until the stream has run the call; nothing
 * is allocated, no state is kept between calls, the device is never synchronised.  Inputs are never written; an output must
 * not overlap an input or another output.  Calls from several host threads on different streams are safe where they share
 * no output and no workspace.  Status codes are attn_status (attn.h); all argument checks run before anything is enqueued.
 * bf16 tensors, weights, tables, caches and workspaces are 16-byte aligned, int and other float arrays 4-byte.
 */
#ifndef PAPER_2605_10905_KV_H
#define PAPER_2605_10905_KV_H

#include "attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * rope_qkv -- split, norm and rotation of a packed projection.
 *   qkv        bfloat16, B * N rows (row b * N + n is token n of sequence b) of (Hq + 2 Hkv) * d features: the query heads,
 *              the key heads, the value heads; consecutive rows are `ld` elements apart (a multiple of 8)
 *   q_weight, k_weight   bfloat16 [d], or both NULL: no norm
 *   eps        >= 0, added to the mean square
 *   table      see above; may be NULL with rot = 0
 *   npos, rot, interleaved   rot: 0 .. d, a multiple of 16
 *   pos        int32 [B * N]: positions; NULL: token n has position n (N <= npos).  A position outside 0 .. npos - 1 makes
 *              the token's rows of q and k NaN
 *   q          bfloat16 [B, Hq, N, d];  k, v  bfloat16 [B, Hkv, N, d]
 *   d          64 or 128 (ATTN_ERR_UNSUPPORTED otherwise)
 * Errors: ATTN_ERR_NULL (a missing pointer, or one weight without the other), ATTN_ERR_SHAPE (non-positive size,
 * Hq % Hkv != 0, ld too small or no multiple of 8, rot outside 0 .. d, N > npos without pos, misaligned pointer),
 * ATTN_ERR_UNSUPPORTED (d; rot no multiple of 16; eps negative or NaN; B * N * (Hq + 2 Hkv) above 2^31 - 1024), ATTN_ERR_LAUNCH.
 */
int rope_qkv(const void* qkv, long long ld, const void* q_weight, const void* k_weight, float eps,
             const float* table, int npos, int rot, int interleaved, const int* pos,
             void* q, void* k, void* v, int B, int Hq, int Hkv, int N, int d, void* stream);

/*
 * rope_qkv_bwd -- gradients of rope_qkv, given those of its outputs (attn_bwd's dq, dk, dv).
 *
 *     g = R(p)^T dz ;  dweight = sum over tokens and heads of g * x r ;  r = 1 / sqrt(mean(x^2) + eps)
 *     dx = r (g weight - x r mean(g weight x r))              (without weights: dx = g)
 *
 *   dq, dk, dv   bfloat16, layouts of q, k, v
 *   qkv, ld      the forward's input (not used without weights); all arguments to pos as for rope_qkv.  A position outside
 *                the table makes the token's gradients of q and k, and the weights' gradients, NaN
 *   dqkv         bfloat16, rows as qkv's, `dld` elements apart, overwritten (elements between the rows are not touched)
 *   dq_weight, dk_weight   float32 [d], overwritten; not used without weights
 *   workspace    rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) bytes; contents on entry are irrelevant, on return
 *                unspecified; not used without weights
 * Deterministic (no atomics).  Two kernels are enqueued, without weights one.  Errors as for rope_qkv.
 */
int rope_qkv_bwd(const void* dq, const void* dk, const void* dv, const void* qkv, long long ld,
                 const void* q_weight, const void* k_weight, float eps,
                 const float* table, int npos, int rot, int interleaved, const int* pos,
                 void* dqkv, long long dld, float* dq_weight, float* dk_weight, float* workspace,
                 int B, int Hq, int Hkv, int N, int d, void* stream);
/* bytes of workspace for that call with weights (0 for non-positive sizes) */
long long rope_qkv_bwd_workspace_bytes(int B, int Hq, int Hkv, int N, int d);

/*
 * The paged cache: k_cache and v_cache are [num_pages, Hkv, page_size, d] each, bfloat16 (ATTN_BF16) or e4m3 bytes
 * (ATTN_FP8_E4M3: the real values are k_descale and v_descale times the codes'; the de-scales are ignored for
 * ATTN_BF16).  page_size is a power of two from 16 to 1024, and W * page_size at most 2^30 (ATTN_ERR_UNSUPPORTED
 * otherwise).  `pages` is int32 [S, W]: key p of sequence s is row p % page_size of page pages[s][p / page_size], for
 * p < W * page_size.
 *
 * kv_append -- new tokens of a serving batch: split, norm and rotation as rope_qkv, into the cache.
 *   qkv .. interleaved   as for rope_qkv, T rows
 *   pos        int32 [T], required: the token's position, by which it is rotated and which names its place in the cache
 *   seq        int32 [T]: its sequence; NULL: token t belongs to sequence t (T <= S)
 *   q          bfloat16 [T, Hq, d]
 * Codes are round-to-nearest-even of value / de-scale, saturated at +-448 (NaN stays NaN).
 * A token with a negative position is padding: nothing is written for it, neither q nor cache.  A token whose position is not
 * below npos (where rot > 0), or whose sequence is outside 0 .. S - 1, gets NaN in its row of q and does not enter the cache; one whose
 * page is outside the table (p >= W * page_size) or whose entry is outside 0 .. num_pages - 1 gets its q and does not enter the cache.
 * Tokens of one call must not name the same place of the cache twice: what it then holds is unspecified, and may be a mix.
 * Nothing else of the cache is touched.  One kernel.  Errors as for rope_qkv, and ATTN_ERR_DTYPE, ATTN_ERR_UNSUPPORTED for a
 * page_size, or with ATTN_FP8_E4M3 for a de-scale outside 2^-96 .. the largest float32.
 */
int kv_append(const void* qkv, long long ld, const void* q_weight, const void* k_weight, float eps,
              const float* table, int npos, int rot, int interleaved, const int* pos, const int* seq, const int* pages,
              void* q, void* k_cache, void* v_cache, int T, int S, int Hq, int Hkv, int d,
              int W, int page_size, int num_pages, int dtype, float k_descale, float v_descale, void* stream);

/*
 * kv_decode -- attention of one token per sequence over the paged cache.
 *
 *     s_j = scale q . k_j ;  o = sum_j exp(s_j) v_j / sum_j exp(s_j) ;  lse = ln sum_j exp(s_j)        j < lens[b]
 *
 *   q          bfloat16 [B, Hq, d] (kv_append's q); query head h reads key head h / (Hq / Hkv)
 *   pages      int32 [B, W];  lens  int32 [B]: keys of each sequence, the new token's own among them (taken as at most
 *              W * page_size).  Keys of an entry outside 0 .. num_pages - 1 are hidden
 *   o          bfloat16 [B, Hq, d];  lse  float32 [B, Hq], required.  A row without visible keys, or all of whose scores are -inf, gets
 *              o = 0, lse = -inf
 *   workspace  kv_decode_workspace_bytes(B, Hq, Hkv, d) bytes; contents on entry are irrelevant, on return unspecified;
 *              calls that can overlap on the device must not share it
 *   scale      > 0; scale * log2(e), with ATTN_FP8_E4M3 times k_descale, has to be a normal float32, and de-scales as for kv_append
 *              (ATTN_ERR_UNSUPPORTED otherwise)
 *   d          64 or 128; B * Hq below 2^24 (ATTN_ERR_UNSUPPORTED otherwise)
 * What lies in the cache behind a sequence's last key, or in pages that no visible key names, is never read into a result.
 * Two kernels are enqueued.  The split of the keys over workgroups is computed on the device from `lens`: the call can be captured once and replayed while
 * the sequences grow.  Deterministic.  Products are taken on bf16 with 32-bit sums (e4m3 values are exact in bf16); softmax
 * statistics and sums are 32 bits; a probability enters the second product as the sum of two bf16, 2^-15 of it off.
 */
int kv_decode(const void* q, const void* k_cache, const void* v_cache, const int* pages, const int* lens,
              void* o, float* lse, void* workspace, int B, int Hq, int Hkv, int d,
              int W, int page_size, int num_pages, float scale, int dtype, float k_descale, float v_descale, void* stream);
long long kv_decode_workspace_bytes(int B, int Hq, int Hkv, int d);

#ifdef __cplusplus
}
#endif
#endif
