// Attention of one new token per sequence over the paged cache (kv_decode).
//
// The call reads every visible key and value once and does 2 G operations on each feature of a key and 4 G on each of a value (G query heads
// share a key head), so it is bound by memory as long as the products run on the matrix cores and enough bytes are in flight.  A wave holds
// 64 queries at most: keys and values are read ceil(G / 64) times.
//
// Measured, where a 1 GiB device copy runs at 5.16 TB/s (keys and values read a second, both kernels): 2 x 131072 keys, 64/8 heads, d = 128
// 188 - 190 us (5.7 TB/s); 64 ragged sequences up to 6000 151 - 152 (5.4); 32 up to 9000, e4m3 65.5 - 66.3 (4.6); 24 up to 1500, 16/16 heads, d = 64
// 20.5 - 21 (3.7); 1 x 500, 32/8 heads 8.2, which is two launches.  Groups of 64 queries, 64 x 4000 keys, 64/1 heads: d = 128 44.7 (2.9), e4m3 31.6
// (2.1); d = 64 24.5 (2.7), e4m3 22.0 (1.5): bound by the vector work of 64 rows, not by memory.
//
// Probabilities enter the second product as two bf16 (see there).  Rounded to one, which put o 19 - 35 % further off the definition, the same calls
// took 187 - 190, 150 - 152, 65.1 - 65.6, 20.2 - 20.6, 8.1; 42.6, 29.0; 22.9, 20.0.  The figures beside the choices below were taken with one: they
// compare the two sides.
//
// Split: the work is the list of all tiles (8 KB of keys: 32, 64 or 128 of them, and their values), sequence by sequence, key head by
// key head; each of kWorkers waves takes an equal, consecutive piece of it, whatever the lengths are.  What the pieces are follows from
// `lens` on the device, by a scan over them that every wave does for itself.  A wave that covers all tiles of a (sequence, key head) writes its
// rows of o; a wave that covers some of them leaves its sums (32 bits) in the workspace, at most two per wave (where its piece begins and
// where it ends), and the second kernel joins them.  Where the four waves of a workgroup work on one (sequence, key head) alone, they add
// their sums in LDS first.
//
// A wave streams its tiles through a ring of its own in LDS (two of 16 KB: 128 KB of a CU's four waves, of which at least half is in
// flight), by direct-to-LDS loads, so that no barrier is needed while it does.  Page entries come through the scalar cache, whose counter is
// not the tiles'.  A block of 16 rows lies in one page (pages hold 16 rows or more).
//
// Products are taken transposed, as in attn_fwd: S^T = K Q^T and O^T += V^T P^T on the 16x16x32 MFMA, the queries of the group as its
// 16 columns (NQ blocks of them, fed by the same keys).  A lane then holds keys 4 g + r of both blocks of 32 keys for one query, which
// are the eight k of its second operand in place: key 4 g + r of block e is k = 8 g + 4 e + r, and V is read (transposing LDS loads)
// in the same order.
#include <type_traits>

#include "attn_device.h"
#include "kv_kernels.h"

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

constexpr int kWaves = 4, kWorkers = 1024, kWorkersLog2 = 10, kWorkgroups = kWorkers / kWaves;
constexpr float kLn2 = 0.6931471805599453f;

// a value that all lanes agree on, in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long x) {
  return (unsigned long long)(uint32_t)uniform((int)(uint32_t)x) | ((unsigned long long)(uint32_t)uniform((int)(x >> 32)) << 32);
}
// scalar load of what no kernel writes while this one runs
__device__ __forceinline__ int scalar_load(const int* p, size_t i) { return ((const __attribute__((address_space(4))) int*)p)[i]; }

__device__ __forceinline__ int visible_keys(const DecodeParams& p, int len) { return min(max(len, 0), p.W << p.page_log2); }

// A tile is 8 KB of keys: 32 rows of 256 bytes, 64 of 128, 128 of 64.  (Tiles of 32 keys throughout cost the same time per tile, about 3000
// cycles of one wave, for a half or a quarter of the bytes: 66 us for 32 ragged e4m3 sequences up to 9000 where the memory needs 57.)
template <int ROWB>
constexpr int kTileLog2 = ROWB == 256 ? 5 : ROWB == 128 ? 6 : 7;
template <int TL>
__device__ __forceinline__ int tiles_of(int keys) {
  return (keys + (1 << TL) - 1) >> TL;
}

// inclusive sums over the lanes: shifts inside rows of 16, then the rows' last sums
__device__ __forceinline__ uint32_t scan64(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);  // row_bcast 15 into rows 1 and 3
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);  // row_bcast 31 into rows 2 and 3
  return x;
}

// Where the piece of wave i begins in a list of `all` tiles: equal pieces; or, where there are fewer tiles than waves, one tile each for the first
// of them, side by side, so that the four of a workgroup can add their sums (1 x 30000 keys, 8/1 heads 19.7 -> 12.6 us); or, where there are no
// more than workgroups, one for each workgroup's first wave (1 x 500, 32/8 heads 7.9 us, side by side 8.7).
__device__ __forceinline__ unsigned long long piece_begin(unsigned long long all, int i) {
  if (all >= kWorkers) return (all * (unsigned)i) >> kWorkersLog2;
  return min((unsigned long long)(unsigned)(all <= kWorkgroups ? (i + kWaves - 1) / kWaves : i), all);
}

// A wave's piece [begin, end) of the list of all tiles, and the sequence that it begins in.
struct Piece {
  unsigned long long all, begin, end;
  int b, len;                 // the sequence and its visible keys
  unsigned long long before;  // tiles of one key head in front of it
};
template <int TL>
__device__ __forceinline__ Piece piece_of(const DecodeParams& p, int worker, int units) {
  constexpr int HELD = 4;  // lengths that a lane holds: batches of 256 are read once, longer ones twice
  const int lane = threadIdx.x & 63;
  Piece r;
  // (a sequence has at most 2^25 tiles of 32 keys: sums over 64 of them fit 32 bits)
  int len[HELD];
  uint32_t incl[HELD];
  unsigned long long total = 0;
#pragma unroll
  for (int c = 0; c < HELD; ++c) len[c] = 64 * c + lane < p.B ? p.lens[64 * c + lane] : 0;
#pragma unroll
  for (int c = 0; c < HELD; ++c) {
    len[c] = visible_keys(p, len[c]);
    incl[c] = 0;
    if (c == 0 || p.B > 64 * c) incl[c] = scan64(tiles_of<TL>(len[c]));
    total += (uint32_t)__builtin_amdgcn_readlane((int)incl[c], 63);
  }
  if (p.B > 64 * HELD) {
    unsigned long long mine = 0;
    for (int b = 64 * HELD + lane; b < p.B; b += 64) mine += tiles_of<TL>(visible_keys(p, p.lens[b]));
#pragma unroll
    for (int m = 1; m < 64; m *= 2) mine += __shfl_xor(mine, m);
    total += uniform(mine);
  }
  r.all = total * (unsigned)units;
  r.begin = piece_begin(r.all, worker);
  r.end = piece_begin(r.all, worker + 1);
  r.b = r.len = 0;
  r.before = 0;
  unsigned long long base = 0;
  // whether the sequence that the piece begins in is behind these 64; if not, it is the last of them that does not begin behind it
  auto behind = [&](int first, int len64, uint32_t incl64) __attribute__((always_inline)) {
    const uint32_t excl = incl64 - tiles_of<TL>(len64);
    const int n = __popcll(__ballot(first + lane < p.B && (base + excl) * (unsigned)units <= r.begin));
    if (n > 0) {
      r.b = first + n - 1;
      r.len = __builtin_amdgcn_readlane(len64, n - 1);
      r.before = base + (uint32_t)__builtin_amdgcn_readlane((int)excl, n - 1);
    }
    base += (uint32_t)__builtin_amdgcn_readlane((int)incl64, 63);
    return n == 64 && first + 64 < p.B;
  };
  bool more = true;
#pragma unroll
  for (int c = 0; c < HELD; ++c)
    if (more) more = behind(64 * c, len[c], incl[c]);
  for (int first = 64 * HELD; more; first += 64) {
    const int next = first + lane < p.B ? visible_keys(p, p.lens[first + lane]) : 0;
    more = behind(first, next, scan64(tiles_of<TL>(next)));
  }
  return r;
}

__device__ __forceinline__ float max_rows(float x) {  // over lanes l, l ^ 16, l ^ 32, l ^ 48
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return attn_max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_rows(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return attn_sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ bf16x8 e4m3_to_bf16(uint32_t lo, uint32_t hi) {  // (exact)
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
  return __builtin_bit_cast(bf16x8, o);
}

// query heads that one unit of the list takes, and units of a sequence
__host__ __device__ constexpr int blocks_for(int G) { return G <= 16 ? 1 : G <= 32 ? 2 : 4; }
__host__ __device__ __forceinline__ int rows_kept(int G) { return G < 16 * blocks_for(G) ? G : 16 * blocks_for(G); }
// floats of one wave's sums: rows of O, then (reference maximum, sum) of each row
template <typename I>
__host__ __device__ __forceinline__ I partial_floats(int rows, I d) {
  return rows * d + (2 * rows + 3) / 4 * 4;
}
// What the second kernel has to know of each (sequence, unit), behind the sums: written by the wave that takes its first tile (first)
// and, where that is another one, by the wave that takes its last (last).
struct Split {
  int first;  // 2 * wave + which of its two sums the first part is; -1: one wave took it all
  int last;   // the wave of the last part
  int ends;   // (with last) whether that wave's piece ends with this (sequence, unit)
  int step;   // (with first) waves from one with a part to the next
};
template <typename I>
__host__ __device__ __forceinline__ size_t split_offset(int rows, I d) {
  return (size_t)2 * kWorkers * partial_floats(rows, d) * sizeof(float);
}

// JOINT: whether a workgroup's waves add their sums where they can (see the end).
template <int D, bool FP8, int NQ, bool JOINT>
__global__ void __launch_bounds__(kWaves * 64, 1) kv_decode_kernel(const DecodeParams p) {
  constexpr int ROWB = D * (FP8 ? 1 : 2), NCH = ROWB / 16, TL = kTileLog2<ROWB>, KT = 1 << TL, TILEB = KT * ROWB;
  constexpr int NB = KT / 16, NP = KT / 32;                    // blocks of 16 keys, pairs of them
  constexpr int LPT = TILEB / 1024, PIECE_ROWS = 1024 / ROWB;  // direct loads of a tile of keys or values, rows of one
  constexpr int LPB = LPT / NB > 0 ? LPT / NB : 1, RING = 2, NDB = D / 16, NKS = D / 32;
  static_assert(TILEB == 8192 && PIECE_ROWS <= 16 && LPB * NB == LPT, "a direct load stays inside a block of 16 keys");
  // The rows of q that a tile is the first to need come with it where they fit the LDS.  (Loaded to registers at the change, they are waited
  // for behind all tiles requested before.  This kernel, us: 24 ragged sequences up to 1500 keys, 16 heads, d = 64 18.6 -> 17.7;
  // 16 x 2000, 32/8 heads 27.0 -> 25.7; 32 ragged e4m3 sequences up to 9000, 64/8 heads 62.9 -> 61.3.)
  constexpr bool QRING = NQ == 1;
  constexpr int QB = QRING ? 32 * D : 0, QLOADS = QB / 1024;
  constexpr int STATB = QRING ? RING * QB : NQ * 16 * 8;  // at the end: (maximum, sum) of the wave's rows
  __shared__ __attribute__((aligned(1024))) char smem_raw[kWaves * (RING * 2 * TILEB + STATB)];
  LDS_AS char* const smem = (LDS_AS char*)smem_raw;

  const int w = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, j16 = lane & 15, g = lane >> 4;
  const int worker = blockIdx.x * kWaves + w;
  const int G = p.Hq / p.Hkv, QG = (G + 16 * NQ - 1) / (16 * NQ), units = p.Hkv * QG;
  const int page_mask = (1 << p.page_log2) - 1;

  const Piece at = piece_of<TL>(p, worker, units);
  if (at.begin == at.end) return;  // (no wave of its workgroup comes to the barrier below then)
  const int n = (int)(at.end - at.begin);  // (2^10 waves share far below 2^41 tiles: a cache fits the memory)

  // A position in the list: tile t of `unit` of sequence b, and the page entries of its blocks
  struct Position {
    int b, unit, t, nt, len, e[NB];
  };
  auto entries = [&](Position& x) __attribute__((always_inline)) {
    const size_t row = (size_t)x.b * p.W;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int j = (x.t << TL) + 16 * i;  // (below len in block 0: there is no tile without keys)
      x.e[i] = scalar_load(p.pages, row + ((i == 0 || j < x.len ? j : x.t << TL) >> p.page_log2));
    }
  };
  auto advance = [&](Position& x) __attribute__((always_inline)) {
    if (++x.t < x.nt) return;
    x.t = 0;
    if (++x.unit < units) return;
    x.unit = 0;
    do {  // (there is another tile: no more are asked for than the list has)
      if (x.b + 1 >= p.B) break;
      ++x.b;
      x.len = visible_keys(p, scalar_load(p.lens, x.b));
    } while (x.len == 0);
    x.nt = tiles_of<TL>(x.len);
  };
  Position ld;
  {
    const unsigned long long rest = at.begin - at.before * (unsigned)units;
    ld.b = at.b;
    ld.len = at.len;
    ld.nt = tiles_of<TL>(at.len);
    if (rest >> 32 == 0) {  // (a quotient of 32 bits is a fifth of one of 64)
      ld.unit = uniform((int)((uint32_t)rest / (uint32_t)ld.nt));
      ld.t = uniform((int)((uint32_t)rest - (uint32_t)ld.unit * (uint32_t)ld.nt));
    } else {
      ld.unit = uniform((int)(rest / (unsigned)ld.nt));
      ld.t = uniform((int)(rest - (unsigned long long)ld.unit * (unsigned)ld.nt));
    }
  }
  Position cp = ld;
  entries(ld);

  // ---- direct loads: piece c of a block is rows c * PIECE_ROWS + lane / NCH; chunks are swizzled on the global side (the swizzles
  // repeat every 16 rows) ----
  uint32_t koff[LPB], voff[LPB];
#pragma unroll
  for (int c = 0; c < LPB; ++c) {
    const int r = c * PIECE_ROWS + lane / NCH, ch = lane % NCH;
    koff[c] = r * ROWB + ((ch ^ attn_swz_k<ROWB>(r)) << 4);
    voff[c] = r * ROWB + ((ch ^ (FP8 ? attn_swz_k<ROWB>(r) : attn_swz_v<ROWB>(r))) << 4);
  }
  uint32_t qoff[QRING ? QLOADS : 1];  // 16 query rows, chunks swizzled as the keys' (rows past the group's last re-read it)
  if constexpr (QRING) {
    constexpr int QCH = D / 8;
#pragma unroll
    for (int c = 0; c < QLOADS; ++c) {
      const int r = c * (64 / QCH) + lane / QCH, ch = lane % QCH;
      qoff[c] = min(r, G - 1) * (D * 2) + ((ch ^ attn_swz_k<D * 2>(r)) << 4);
    }
  }
  const uint32_t wave_base = w * (RING * 2 * TILEB), ring = (uint32_t)(uintptr_t)smem + wave_base;
  const uint32_t q_base = kWaves * RING * 2 * TILEB + w * (RING * QB), q_ring = (uint32_t)(uintptr_t)smem + q_base;
  bool ld_first = true;
  // Requests tile `ld` into `slot`; bit i of the result: block i has a page and a key.  A block that has none is read from where the tile
  // begins (or the cache's first rows) and hidden later.
  auto issue = [&](int slot) __attribute__((always_inline)) {
    const int j0 = ld.t << TL, hk = ld.unit / QG;
    size_t from[NB];
    uint32_t ok = 0;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const bool has = (unsigned)ld.e[i] < (unsigned)p.num_pages;
      from[i] = has ? ((((size_t)ld.e[i] * p.Hkv + hk) << p.page_log2) + ((j0 + (j0 + 16 * i < ld.len ? 16 * i : 0)) & page_mask)) * ROWB : 0;
      ok |= has && j0 + 16 * i < ld.len ? 1u << i : 0u;
    }
    // Pieces behind the last key read the tile's first rows once more, which are in the caches (1000 ragged sequences up to 60
    // keys, 32/8 heads 55.8 -> 51.3 us; long ones are not slower).
    auto at_piece = [&](int c) __attribute__((always_inline)) {
      const size_t other = from[0] - (size_t)((c % LPB) * PIECE_ROWS * ROWB);
      return c % LPB > 0 && j0 + c * PIECE_ROWS >= ld.len ? other : from[c / LPB];
    };
    const uint32_t to = ring + slot * (2 * TILEB);
    if constexpr (QRING) {
      if (ld.t == 0 || ld_first) {
        const char* const q_rows = (const char*)p.q + ((size_t)ld.b * p.Hq + (size_t)hk * G) * (D * 2);
#pragma unroll
        for (int c = 0; c < QLOADS; ++c) attn_lds_dma16(q_rows, qoff[c], q_ring + slot * QB + c * 1024);
      }
      ld_first = false;
    }
#pragma unroll
    for (int c = 0; c < LPT; ++c) attn_lds_dma16((const char*)p.k + at_piece(c), koff[c % LPB], to + c * 1024);
#pragma unroll
    for (int c = 0; c < LPT; ++c) attn_lds_dma16((const char*)p.v + at_piece(c), voff[c % LPB], to + TILEB + c * 1024);
    return ok;
  };

  // ---- operand addresses in slot 0, first block or pair ----
  constexpr int NKR = FP8 ? D / 64 : NKS;  // 16-byte reads of a key row: e4m3 rows hold two k-steps in one
  uint32_t ka[NKR], va[NDB][2];
#pragma unroll
  for (int s = 0; s < NKR; ++s) ka[s] = wave_base + j16 * ROWB + (((4 * s + g) ^ attn_swz_k<ROWB>(j16)) << 4);
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (FP8) {  // eight rows of one column: 4 g .. 4 g + 3 of both blocks
        const int i = j16 >> 1, r = (i < 4 ? 0 : 16) + 4 * g + (i & 3);
        va[db][e] = wave_base + TILEB + r * ROWB + ((db ^ attn_swz_k<ROWB>(r)) << 4) + ((j16 & 1) << 3);
      } else {  // four rows, 4 g .. 4 g + 3 of block e
        const int r = 16 * e + 4 * g + (j16 >> 2);
        va[db][e] = wave_base + TILEB + r * ROWB + (((2 * db + ((j16 & 3) >> 1)) ^ attn_swz_v<ROWB>(r)) << 4) + ((j16 & 1) << 3);
      }
    }

  bf16x8 q[NQ][NKS];
  f32x4 o[NQ][NDB];
  float m[NQ], l[NQ];
  // features of step s that a lane holds, in chunks of 8
  auto q_chunk = [&](int s) __attribute__((always_inline)) { return FP8 ? 8 * (s >> 1) + 2 * g + (s & 1) : 4 * s + g; };
  auto start = [&](int slot) __attribute__((always_inline)) {  // the rows of cp's unit
    const int hk = cp.unit / QG, first = (cp.unit - hk * QG) * 16 * NQ;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      if constexpr (QRING) {
#pragma unroll
        for (int s = 0; s < NKS; ++s)
          q[i][s] = __builtin_bit_cast(bf16x8, *(LDS_AS u32x4*)(smem + q_base + slot * QB + j16 * (D * 2) + ((q_chunk(s) ^ attn_swz_k<D * 2>(j16)) << 4)));
      } else {
        const int h = first + 16 * i + j16;
        const char* const src = (const char*)p.q + ((size_t)cp.b * p.Hq + (size_t)hk * G + h) * (D * 2);
#pragma unroll
        for (int s = 0; s < NKS; ++s) q[i][s] = __builtin_bit_cast(bf16x8, h < G ? *(const u32x4*)(src + q_chunk(s) * 16) : u32x4{0, 0, 0, 0});
      }
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[i][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[i] = -__builtin_inff();
      l[i] = 0.f;
    }
  };
  const int kept = rows_kept(G);
  // what the second kernel has to know, by the wave with the first tile (head) and the one with the last (tail)
  auto record = [&](bool head, bool tail, bool whole, int part, bool ends) __attribute__((always_inline)) {
    if (lane != 0 || !(head || tail)) return;
    Split* const x = (Split*)((char*)p.ws + split_offset(kept, D)) + ((size_t)cp.b * units + cp.unit);
    if (head) {
      x->first = whole ? -1 : 2 * worker + part;
      x->step = at.all <= kWorkgroups ? kWaves : 1;
    }
    if (tail && !whole) {
      x->last = worker;
      x->ends = ends ? 1 : 0;
    }
  };
  auto finish = [&](bool head, bool tail, int part, bool ends) __attribute__((always_inline)) {  // (with the first tile, with the last)
    const int hk = cp.unit / QG, first = (cp.unit - hk * QG) * 16 * NQ;
    const bool whole = head && tail;
    record(head, tail, whole, part, ends);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int r = 16 * i + j16;
      const float sum = sum_rows(l[i]);
      if (first + r >= G) continue;
      if (whole) {
        const size_t row = (size_t)cp.b * p.Hq + (size_t)hk * G + first + r;
        const float inv = sum == 0.f ? 0.f : p.out_scale / sum;
        char* const dst = (char*)p.o + row * (D * 2) + g * 8;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
          *(u32x2*)(dst + db * 32) = u32x2{attn_pack_bf16(o[i][db][0] * inv, o[i][db][1] * inv), attn_pack_bf16(o[i][db][2] * inv, o[i][db][3] * inv)};
        if (g == 0) p.lse[row] = sum == 0.f ? -__builtin_inff() : (m[i] * p.scale_log2 + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        float* const dst = (float*)p.ws + (size_t)(2 * worker + part) * partial_floats(kept, D);
#pragma unroll
        for (int db = 0; db < NDB; ++db) *(f32x4*)(dst + r * D + db * 16 + g * 4) = o[i][db];
        if (g == 0) {
          dst[kept * D + 2 * r] = m[i];
          dst[kept * D + 2 * r + 1] = sum;
        }
      }
    }
  };
  // waits until at most N loads of this tile are under way (and those of the tile behind it, where one is requested: 2 LPT of them; with
  // rows of q in front of it more, so that a few of its own are then waited for)
  auto wait = [&](auto value, bool behind) __attribute__((always_inline)) {
    constexpr int N = decltype(value)::value;
    if (behind) ATTN_WAIT_VMCNT(2 * LPT + N);
    else ATTN_WAIT_VMCNT(N);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  uint32_t have = 0;  // NB bits for each tile in the ring
  int began = cp.t, slot = 0, part = 0;
  bool fresh = true;
  if constexpr (!QRING) start(0);
  for (int i = 0; i < min(n, RING); ++i) {
    have |= issue(i) << (NB * i);
    if (i + 1 < n) {
      advance(ld);
      entries(ld);
    }
  }
  for (int i = 0; i < n; ++i) {
    const int base = slot * (2 * TILEB);
    const bool behind = i + 1 < n;
    wait(std::integral_constant<int, LPT>{}, behind);
    if constexpr (QRING) {
      if (fresh) start(slot);
      fresh = false;
    }

    // visible rows of the tile's blocks
    const int keys = cp.len - (cp.t << TL);
    auto rows = [&](int e) __attribute__((always_inline)) { return have >> e & 1 ? min(keys - 16 * e, 16) : 0; };
    const bool hidden = keys < KT || (have & ((1u << NB) - 1)) != (1u << NB) - 1;

    f32x4 s[NQ][NB];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
      bf16x8 k[NKS];
#pragma unroll
      for (int x = 0; x < NKR; ++x) {
        const u32x4 c = *(LDS_AS u32x4*)(smem + ka[x] + base + e * 16 * ROWB);
        if constexpr (FP8) {
          k[2 * x] = e4m3_to_bf16(c[0], c[1]);
          k[2 * x + 1] = e4m3_to_bf16(c[2], c[3]);
        } else {
          k[x] = __builtin_bit_cast(bf16x8, c);
        }
      }
#pragma unroll
      for (int i2 = 0; i2 < NQ; ++i2) {
        s[i2][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NKS; ++x) s[i2][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[x], q[i2][x], s[i2][e], 0, 0, 0);
      }
    }
    if (hidden) {
#pragma unroll
      for (int e = 0; e < NB; ++e)
#pragma unroll
        for (int i2 = 0; i2 < NQ; ++i2)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * g + r >= rows(e)) s[i2][e][r] = -__builtin_inff();
    }

    // streaming softmax; differences are taken before they are scaled, so that scores near the type's lowest value do not overflow
    bf16x8 pr[NQ][NP], rest[NQ][NP];
#pragma unroll
    for (int i2 = 0; i2 < NQ; ++i2) {
      float mx = s[i2][0][0];
#pragma unroll
      for (int x = 1; x < 4 * NB; ++x) mx = fmaxf(mx, s[i2][x >> 2][x & 3]);
      const float m_new = fmaxf(m[i2], max_rows(mx)), ref = m_new == -__builtin_inff() ? 0.f : m_new;
      if (__any(m_new != m[i2])) {
        const float alpha = __builtin_amdgcn_exp2f((m[i2] - ref) * p.scale_log2);
#pragma unroll
        for (int db = 0; db < NDB; ++db) o[i2][db] *= alpha;
        l[i2] *= alpha;
      }
      m[i2] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        float e[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          e[y] = __builtin_amdgcn_exp2f((s[i2][2 * x + (y >> 2)][y & 3] - ref) * p.scale_log2);
          sum += e[y];
        }
        // bf16 for the matrix cores, in two parts: the first eight bits of a probability, and the rest, itself rounded (at most 2^-7 of it,
        // so off by 2^-15).  2^-18 of it more, so that both parts are positive, as numbers of bf16 above 2^-108, and an infinite value stays one.
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float e0 = e[2 * y], e1 = e[2 * y + 1], h0 = __uint_as_float(__float_as_uint(e0) & 0xffff0000u), h1 = __uint_as_float(__float_as_uint(e1) & 0xffff0000u);
          hi[y] = __builtin_amdgcn_perm(__float_as_uint(e1), __float_as_uint(e0), 0x07060302u);
          lo[y] = attn_pack_bf16(fmaf(e0, 1.f + 0x1p-18f, -h0), fmaf(e1, 1.f + 0x1p-18f, -h1));
        }
        pr[i2][x] = __builtin_bit_cast(bf16x8, u32x4{hi[0], hi[1], hi[2], hi[3]});
        rest[i2][x] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], lo[2], lo[3]});
      }
      l[i2] += sum;  // (of the unrounded probabilities, this lane's keys)
    }

    wait(std::integral_constant<int, 0>{}, behind);
    if (hidden) {  // 0 times what lies in a hidden row would be NaN where that is not finite
#pragma unroll
      for (int c = 0; c < LPT; ++c) {
        const int r = (c % LPB) * PIECE_ROWS + lane / NCH;
        if (r >= rows(c / LPB)) *(LDS_AS u32x4*)(smem + wave_base + base + TILEB + c * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int x = 0; x < NP; ++x)
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        bf16x8 v;
        const int at_pair = base + x * 32 * ROWB;
        if constexpr (FP8) {
          const i32x2 c = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_AS i32x2*)(smem + va[db][0] + at_pair));
          v = e4m3_to_bf16((uint32_t)c[0], (uint32_t)c[1]);
        } else {
          const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(smem + va[db][0] + at_pair));
          const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(smem + va[db][1] + at_pair));
          v = __builtin_bit_cast(bf16x8, s16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
        }
#pragma unroll
        for (int i2 = 0; i2 < NQ; ++i2) {
          o[i2][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, rest[i2][x], o[i2][db], 0, 0, 0);
          o[i2][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pr[i2][x], o[i2][db], 0, 0, 0);
        }
      }

    // the slot is free once its last operand has arrived
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    have >>= NB;
    if (i + RING < n) {
      have |= issue(slot) << (NB * (RING - 1));
      if (i + RING + 1 < n) {
        advance(ld);
        entries(ld);
      }
    }
    slot ^= 1;

    const bool last = cp.t + 1 == cp.nt;
    if (JOINT && i + 1 == n) break;
    if (last || i + 1 == n) {
      finish(began == 0, last, part, i + 1 == n);
      part = 1;
      if (i + 1 < n) {
        advance(cp);
        if constexpr (!QRING) start(0);
        fresh = true;
        began = 0;
      }
    } else {
      ++cp.t;
    }
  }
  if constexpr (!JOINT) return;

  // Whether the pieces of the workgroup's waves lie in this (sequence, unit): then all of them find so, and add their sums.
  const unsigned long long seg_begin = at.end - 1 - (unsigned)cp.t, seg_end = seg_begin + (unsigned)cp.nt;
  // (Not where one of them has no tile: the end of the workgroup's pieces then lies behind the list, or there are no more tiles than workgroups.)
  const unsigned long long wg_begin = piece_begin(at.all, worker - w);
  const unsigned long long wg_end = at.all < kWorkers ? (unsigned)(worker - w + kWaves) : piece_begin(at.all, worker - w + kWaves);
  if (at.all <= kWorkgroups || wg_begin < seg_begin || seg_end < wg_end) {
    finish(began == 0, cp.t + 1 == cp.nt, part, true);
    return;
  }

  // The workgroup's sums: every wave leaves its own in its ring and adds a quarter of the blocks of all four, in the waves' order: four times
  // fewer parts to write, read and join.
  const bool head = seg_begin == wg_begin, tail = wg_end == seg_end, whole = head && tail;
  record(head && w == 0, tail && w == kWaves - 1, whole, 0, true);
  auto stat = [&](int wave) __attribute__((always_inline)) { return (LDS_AS float*)(smem + kWaves * RING * 2 * TILEB + wave * STATB); };
  auto block = [&](int wave, int x) __attribute__((always_inline)) { return (LDS_AS f32x4*)(smem + wave * (RING * 2 * TILEB) + (x * 64 + lane) * 16); };
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const float sum = sum_rows(l[i]);
    if (g == 0) {
      stat(w)[2 * (16 * i + j16)] = m[i];
      stat(w)[2 * (16 * i + j16) + 1] = sum;
    }
#pragma unroll
    for (int db = 0; db < NDB; ++db) *block(w, i * NDB + db) = o[i][db];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    float wm[kWaves], mx = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      wm[k] = stat(k)[2 * (16 * i + j16)];
      mx = fmaxf(mx, wm[k]);
    }
    const float ref = mx == -__builtin_inff() ? 0.f : mx;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      wm[k] = __builtin_amdgcn_exp2f((wm[k] - ref) * p.scale_log2);
      sum += wm[k] * stat(k)[2 * (16 * i + j16) + 1];
    }
    const int hk = cp.unit / QG, first = (cp.unit - hk * QG) * 16 * NQ, r = 16 * i + j16;
    const size_t row = (size_t)cp.b * p.Hq + (size_t)hk * G + first + r;
    const float inv = sum == 0.f ? 0.f : p.out_scale / sum;
    float* const dst = (float*)p.ws + (size_t)(2 * (worker - w)) * partial_floats(kept, D);
#pragma unroll
    for (int d0 = 0; d0 < NDB; d0 += kWaves) {
      const int db = d0 + w;
      f32x4 val = *block(0, i * NDB + db) * wm[0];
#pragma unroll
      for (int k = 1; k < kWaves; ++k) val += *block(k, i * NDB + db) * wm[k];
      if (first + r >= G) continue;
      if (whole) *(u32x2*)((char*)p.o + row * (D * 2) + db * 32 + g * 8) = u32x2{attn_pack_bf16(val[0] * inv, val[1] * inv), attn_pack_bf16(val[2] * inv, val[3] * inv)};
      else *(f32x4*)(dst + r * D + db * 16 + g * 4) = val;
    }
    if (w != 0 || g != 0 || first + r >= G) continue;
    if (whole) {
      p.lse[row] = sum == 0.f ? -__builtin_inff() : (mx * p.scale_log2 + __builtin_amdgcn_logf(sum)) * kLn2;
    } else {
      dst[kept * D + 2 * r] = mx;
      dst[kept * D + 2 * r + 1] = sum;
    }
  }
}

// Joins what the waves left of a (sequence, unit) that more than one of them took, or writes the rows of a sequence without keys.  D / 4 lanes
// take a row.  Few parts: they take them one after the other, four requested at a time, and the workgroup's lanes hold different rows; many
// (MANY): different parts of a row are shared out, over a whole workgroup of sixteen waves for each row.  `shares` workgroups
// take a pair.
template <int D, bool MANY, bool JOINT>
__global__ void __launch_bounds__(MANY ? 1024 : 256) kv_join_kernel(const DecodeParams p, int NQ, int shares) {
  constexpr int LPR = D / 4, PER = 64 / LPR, AT_ONCE = 4;  // lanes of a row, rows (MANY: parts) a wave holds side by side
  const int G = p.Hq / p.Hkv, QG = (G + 16 * NQ - 1) / (16 * NQ), units = p.Hkv * QG, kept = rows_kept(G);
  const int segment = shares == 1 ? blockIdx.x : blockIdx.x / shares, b = segment / units, unit = segment - b * units;
  const int* const split = (const int*)((const char*)p.ws + split_offset(kept, D)) + (size_t)segment * 4;
  const int len = visible_keys(p, scalar_load(p.lens, b));
  const int split_first = scalar_load(split, 0), w1 = scalar_load(split, 1), ends = JOINT ? scalar_load(split, 2) : 0;
  const int step = scalar_load(split, 3) == kWaves ? kWaves : 1;
  if (len > 0 && split_first < 0) return;  // one wave took it all
  const int lane = threadIdx.x & 63, w = uniform((int)(threadIdx.x >> 6)), sub = lane / LPR, col = (lane % LPR) * 4;
  const int hk = unit / QG, first_row = (unit - hk * QG) * 16 * NQ, rows = min(kept, G - first_row);
  const size_t out = (size_t)b * p.Hq + (size_t)hk * G + first_row;

  // (kept inside the workspace whatever it holds: `lens` may have changed under the call)
  const int first_sum = min(split_first, 2 * kWorkers - 1), w0 = first_sum >> 1, stride = partial_floats(kept, D);
  // The parts: of every wave from w0 to w1, but one of each workgroup whose four waves work on nothing else (groups g0 to g1).
  const int g0 = (w0 + (first_sum & 1) + kWaves - 1) / kWaves, g1 = (w1 + (ends ? 1 : 0)) / kWaves - 1, groups = JOINT && step == 1 ? max(g1 - g0 + 1, 0) : 0;
  const int front = groups ? kWaves * g0 - w0 : kWorkers;
  const int parts = len == 0 ? 0 : min((w1 - w0) / step + 1 - (kWaves - 1) * groups, kWorkers);  // (without keys there is none)
  auto sums_of = [&](int i) __attribute__((always_inline)) {  // which of the 2 * kWorkers sums part i is
    if (i == 0) return first_sum;
    const int x = !JOINT || i < front ? w0 + i * step : i < front + groups ? kWaves * (g0 + i - front) : w0 + i + (kWaves - 1) * groups;
    return min(2 * x, 2 * kWorkers - 1);
  };

  f32x4 o;
  float m, l;
  auto merge = [&](float om, float ol, const f32x4& oo) __attribute__((always_inline)) {
    const float m_new = fmaxf(m, om), ref = m_new == -__builtin_inff() ? 0.f : m_new;
    const float a = __builtin_amdgcn_exp2f((m - ref) * p.scale_log2), c = __builtin_amdgcn_exp2f((om - ref) * p.scale_log2);
    o = o * a + oo * c;
    l = l * a + ol * c;
    m = m_new;
  };
  // parts i0, i0 + step, ... of row r
  auto add_parts = [&](int r, int i0, int step, int rounds) __attribute__((always_inline)) {
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -__builtin_inff();
    l = 0.f;
    for (int at = i0; at < parts; at += rounds) {
      f32x4 po[AT_ONCE];
      float pm[AT_ONCE], pl[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const float* const src = (const float*)p.ws + (size_t)sums_of(min(at + k * step, parts - 1)) * stride;
        po[k] = *(const f32x4*)(src + r * D + col);
        pm[k] = src[kept * D + 2 * r];
        pl[k] = src[kept * D + 2 * r + 1];
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k)
        if (at + k * step < parts) merge(pm[k], pl[k], po[k]);
    }
  };
  auto write = [&](int r) __attribute__((always_inline)) {
    const float inv = l == 0.f ? 0.f : p.out_scale / l;
    *(u32x2*)((char*)p.o + ((out + r) * D + col) * 2) = u32x2{attn_pack_bf16(o[0] * inv, o[1] * inv), attn_pack_bf16(o[2] * inv, o[3] * inv)};
    if (col == 0) p.lse[out + r] = l == 0.f ? -__builtin_inff() : (m * p.scale_log2 + __builtin_amdgcn_logf(l)) * kLn2;
  };

  if constexpr (!MANY) {
    const int r = (blockIdx.x - segment * shares) * (blockDim.x / LPR) + w * PER + sub;
    if (r >= rows) return;
    add_parts(r, 0, 1, AT_ONCE);
    write(r);
  } else {
    __shared__ float so[16][D], sm[16], sl[16];
    const int r = blockIdx.x - segment * shares;
    if (r >= rows) return;
    add_parts(r, w * PER * AT_ONCE + sub, PER, 16 * PER * AT_ONCE);
#pragma unroll
    for (int k = LPR; k < 64; k *= 2) {
      const float om = __shfl_xor(m, k), ol = __shfl_xor(l, k);
      f32x4 oo;
#pragma unroll
      for (int i = 0; i < 4; ++i) oo[i] = __shfl_xor(o[i], k);
      merge(om, ol, oo);
    }
    if (sub == 0) *(f32x4*)&so[w][col] = o;
    if (lane == 0) {
      sm[w] = m;
      sl[w] = l;
    }
    __syncthreads();
    if (w != 0) return;
    for (int k = 1; k < min(16, (parts + PER * AT_ONCE - 1) / (PER * AT_ONCE)); ++k) merge(sm[k], sl[k], *(const f32x4*)&so[k][col]);
    if (sub == 0) write(r);
  }
}

// Workgroups add their sums where there are few enough (sequence, unit) pairs, on average two workgroups or more to each.  us, apart / added:
// 64 x 4000 keys, 64/1 heads 61.2 / 44.8 (42.5 with the join's rows over more workgroups), 32/1 41.2 / 32.9; 128 x 4000, 32/2 heads 100 / 95; 1 x 131072 e4m3, 8/1 heads 23.1 / 17.3; 2 x 131072,
// 64/8 heads 191.9 / 190.2.  Where it is seldom possible the code for it costs: 211 ragged sequences up to 140 keys, 32/4 heads 17.5 / 18.2;
// 71 up to 1894, e4m3, 56/8 heads 23.8 / 24.3.
bool sums_are_added(long long segments) { return segments <= 128; }

template <int D, bool FP8, bool JOINT>
void launch_decode(const DecodeParams& p, int nq, hipStream_t stream) {
  constexpr int grid = kWorkers / kWaves;
  if (nq == 1) kv_decode_kernel<D, FP8, 1, JOINT><<<grid, kWaves * 64, 0, stream>>>(p);
  else if (nq == 2) kv_decode_kernel<D, FP8, 2, JOINT><<<grid, kWaves * 64, 0, stream>>>(p);
  else kv_decode_kernel<D, FP8, 4, JOINT><<<grid, kWaves * 64, 0, stream>>>(p);
}

template <int D, bool JOINT>
void launch_join(const DecodeParams& p, int nq, int segments, hipStream_t stream) {
  const int kept = rows_kept(p.Hq / p.Hkv), rows_per_wave = 256 / D, waves = (kept + rows_per_wave - 1) / rows_per_wave;
  // Up to 256 / segments parts of each and six more.  us, one part after the other / shared out: 1 x 500 keys, 32/8 heads (8 pairs) 9.6 / 7.9;
  // 2 x 131072, 64/8 (16) 189.4 / 187.5; 14 x 4582 e4m3, 8/2 (28) 15.3 / 14.0; 56 x 900, 8/1 12.8 / 13.6; 100 x 300, 8/1 11.4 / 14.5.
  if constexpr (JOINT) {
    if (segments < 40) {
      kv_join_kernel<D, true, true><<<segments * kept, 1024, 0, stream>>>(p, nq, kept);
      return;
    }
  }
  const int used = waves < 4 ? waves : 4, shares = (kept + used * rows_per_wave - 1) / (used * rows_per_wave);
  kv_join_kernel<D, false, JOINT><<<segments * shares, 64 * used, 0, stream>>>(p, nq, shares);
}

template <bool JOINT>
int launch(const DecodeParams& p, int d, bool fp8, int nq, int segments, hipStream_t stream) {
  if (d == 128 && fp8) launch_decode<128, true, JOINT>(p, nq, stream);
  else if (d == 128) launch_decode<128, false, JOINT>(p, nq, stream);
  else if (fp8) launch_decode<64, true, JOINT>(p, nq, stream);
  else launch_decode<64, false, JOINT>(p, nq, stream);
  if (hipGetLastError() != hipSuccess) return 1;
  if (d == 128) launch_join<128, JOINT>(p, nq, segments, stream);
  else launch_join<64, JOINT>(p, nq, segments, stream);
  return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace

int kv_decode_launch(const DecodeParams& p, int d, bool fp8, hipStream_t stream) {
  const int G = p.Hq / p.Hkv, nq = blocks_for(G), segments = p.B * p.Hkv * ((G + 16 * nq - 1) / (16 * nq));  // (B * Hq fits 24 bits)
  return sums_are_added(segments) ? launch<true>(p, d, fp8, nq, segments, stream) : launch<false>(p, d, fp8, nq, segments, stream);
}

long long kv_decode_bytes(int B, int Hq, int Hkv, int d) {  // (of any sizes, those that no call takes among them)
  const int G = Hq / Hkv, nq = blocks_for(G);
  const long long segments = (long long)B * (Hkv * ((G - 1) / (16 * nq) + 1ll)), most = 1 << 24;  // (no call has more)
  return (long long)split_offset(rows_kept(G), (long long)d) + (segments < most ? segments : most) * (long long)sizeof(Split);
}
