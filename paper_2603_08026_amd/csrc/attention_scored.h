// Attention of listed rows over pages or [B, L] caches with masked and reshaped scores (dyllm_scores): work items, the masks' limits, and the two
// bf16 kernels.
//
// Causal order of blocks, prefixes and the length of a sequence are one number for a row, the limit below which its keys count, because all of
// them hide a tail.  So a tile of keys either lies below the least limit of a wave's rows (no test), or is tested key by key, or lies behind
// the largest (not visited).  Documents hide both ends: the first and the last key with a number between the least and the largest of the
// rows' bound the sweep, and in between a vote over a tile's 32 numbers says whether any test is needed.
#pragma once
#include "attention_common.h"
#include <type_traits>

namespace dy {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// scores as they are; reshaped (cap, slopes); documents too
enum ScoreMode { PLAIN = 0, SHAPED = 1, DOCS = 2 };
inline ScoreMode mode_of(const ScoredAttn &a) { return a.doc ? DOCS : a.soft_cap > 0.f || a.slopes ? SHAPED : PLAIN; }

__device__ __forceinline__ int keys_of(const ScoredAttn &a, int b) { return a.kv_len ? min(max(a.kv_len[b], 0), a.L) : a.L; }

// keys [0, limit) count for a row at position i of sequence b, which has n keys
__device__ __forceinline__ int limit_of(const ScoredAttn &a, int b, int n, int i) {
  if (a.block <= 0) return n;
  const long up = ((long)max(i, 0) / a.block + 1) * a.block;
  const int upto = (int)min((long)n, up);
  return a.prefix ? max(upto, min(a.prefix[b], n)) : upto;
}
// position of row j of sequence b
__device__ __forceinline__ int position_of(const ScoredAttn &a, bool pages, int b, int j) {
  return pages ? a.at[j] : (a.at ? a.at[j] : j) - b * a.L;
}

// ---- work items: (key-value head, sequence, key split, tile of packed rows) ---------------------------------------
// The rows of a sequence and the g heads of a group are packed as in the grouped form above.  Where rows are few the keys of a sequence are split so
// that about `target` workgroups share all keys evenly, whatever the lengths (which the device knows): with W = sum of tiles * keys
// over the sequences, a split has W * Hkv / target keys, and a sequence as many splits as that makes of its keys.
constexpr int SPLIT_KEYS = 128;  // keys that the waves of a workgroup take at a time; a split has a multiple
inline long scored_tiles(const ScoredAttn &a) {  // at most, of one key-value head
  const long g = a.H / a.Hkv;
  return a.offsets ? (a.cap * g + a.bq - 1) / a.bq + a.B : a.B * ((a.L * g + a.bq - 1) / a.bq);
}
inline long scored_items(const ScoredAttn &a) {
  return scored_tiles(a) + (a.splits > 1 ? (a.target + a.Hkv - 1) / a.Hkv : 0);
}
// Which of the 8 XCDs takes which item: the tiles that read one (sequence, head)'s keys stay on as few as the heads allow, next to each other in time.
inline long scored_grid(const ScoredAttn &a) {
  const long t = scored_items(a);
  if (a.Hkv % ATTN_XCD == 0) return t * a.Hkv;
  if (ATTN_XCD % a.Hkv == 0) return (t * a.Hkv + ATTN_XCD - 1) / ATTN_XCD * ATTN_XCD;
  return (t * a.Hkv + ATTN_XCD - 1) / ATTN_XCD * ATTN_XCD;
}
struct ScoredItem {
  int seq = -1, row = 0, packed = 0, n = 0;  // as AttnItem
  int kv_head = 0, keys = 0, split = 0, splits = 1, chunk = 0;
};
__device__ __forceinline__ ScoredItem scored_item(const ScoredAttn &a, int p) {
  const int g = a.H / a.Hkv, lane = threadIdx.x % WAVE, BQ = a.bq;
  ScoredItem it;
  const int total = a.offsets ? min(a.offsets[a.B], a.cap) : a.B * a.L;
  int lo = 0, hi = 0, tiles = 0, keys = 0;
  auto look = [&](int b0) {  // this lane's sequence
    const int b = b0 + lane;
    lo = hi = tiles = keys = 0;
    if (b < a.B) {
      lo = a.offsets ? min(max(a.offsets[b], 0), total) : b * a.L;
      hi = a.offsets ? max(min(a.offsets[b + 1], total), lo) : lo + a.L;
      tiles = ((hi - lo) * g + BQ - 1) / BQ;
      keys = keys_of(a, b);
    }
  };
  int chunk = 0x7fffff80;
  if (a.splits > 1) {
    float w = 0.f;
    for (int b0 = 0; b0 < a.B; b0 += WAVE) {
      look(b0);
      w += (float)tiles * (float)keys;
    }
    w = wave_sum(w) * (float)a.Hkv / (float)a.target;  // (the order of additions is fixed: every workgroup has the same)
    chunk = (int)fminf(w, 1e9f) / SPLIT_KEYS * SPLIT_KEYS + SPLIT_KEYS;
  }
  auto splits_of = [&](int *size) {
    const int least = ((keys + a.splits - 1) / a.splits + SPLIT_KEYS - 1) / SPLIT_KEYS * SPLIT_KEYS;
    *size = max(chunk, least);
    return max(1, (int)(((long)keys + *size - 1) / *size));
  };
  int size = 0, upto = 0, n_items = 0;
  for (int b0 = 0; b0 < a.B; b0 += WAVE) {
    if (a.B > WAVE || a.splits == 1) look(b0);
    upto = wave_scan(tiles * splits_of(&size));
    n_items += __builtin_amdgcn_readlane(upto, WAVE - 1);
  }
  const int x = p % ATTN_XCD, s = p / ATTN_XCD;
  int w;
  if (n_items == 0) return it;
  if (a.Hkv % ATTN_XCD == 0) {
    const int per = a.Hkv / ATTN_XCD;
    if (s / n_items >= per) return it;
    it.kv_head = x * per + s / n_items;
    w = s % n_items;
  } else if (ATTN_XCD % a.Hkv == 0) {
    const int per = ATTN_XCD / a.Hkv;
    it.kv_head = x / per;
    w = s * per + x % per;
    if (w >= n_items) return it;
  } else {
    const long items = (long)n_items * a.Hkv, per_xcd = (items + ATTN_XCD - 1) / ATTN_XCD, at = x * per_xcd + s;
    if (s >= per_xcd || at >= items) return it;
    it.kv_head = (int)(at / n_items);
    w = (int)(at % n_items);
  }
  for (int b0 = 0; b0 < a.B; b0 += WAVE) {
    if (a.B > WAVE) {
      look(b0);
      upto = wave_scan(tiles * splits_of(&size));
    }
    const uint64_t past = __ballot(upto > w);
    if (past) {
      const int f = __ffsll((unsigned long long)past) - 1;
      const int nt = __builtin_amdgcn_readlane(tiles, f), rows = __builtin_amdgcn_readlane(hi - lo, f);
      it.seq = b0 + f;
      it.row = __builtin_amdgcn_readlane(lo, f);
      it.keys = __builtin_amdgcn_readlane(keys, f);
      it.chunk = __builtin_amdgcn_readlane(size, f);
      it.splits = max(1, (int)(((long)it.keys + it.chunk - 1) / it.chunk));
      const int mine = w - (__builtin_amdgcn_readlane(upto, f) - nt * it.splits);
      it.split = mine / nt;
      it.packed = (nt - 1 - mine % nt) * BQ;  // the last rows of a causal sequence have the most keys: they come first
      it.n = min(BQ, rows * g - it.packed);
      return it;
    }
    w -= __builtin_amdgcn_readlane(upto, WAVE - 1);
  }
  return it;
}

// ---- shared pieces of the bf16 kernels -----------------------------------------------------------------------
template <typename V> __device__ __forceinline__ void here(V &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ const unsigned char *uniform_bytes(const void *p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (const unsigned char *)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int wave_min_i(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, WAVE));
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max_i(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, WAVE));
  return __builtin_amdgcn_readfirstlane(v);
}

// Where the keys and values of a sequence and head lie.  A tile of 32 keys starts at a multiple of 32, pages hold a multiple of 16: its two halves
// lie each in one piece.  PAGED: their pages are asked for through the scalar cache, a tile ahead.
template <bool PAGED, int DH> struct KeyPlaces {
  const unsigned char *k, *v;             // of key 0 (pages: of page 0)
  uint32_t stride;                        // bytes from one key to the next
  const __attribute__((address_space(4))) int32_t *table;
  size_t page_bytes;
  int shift, n_pages, bad = 0;
  int ahead[2];                           // pages of the tile asked for
  __device__ __forceinline__ KeyPlaces(const ScoredAttn &a, int b, int kvh) {
    if constexpr (PAGED) {
      const size_t head = ((size_t)kvh << a.pages.shift) * DH * 2;
      k = uniform_bytes((const unsigned char *)a.pages.k + head);
      v = uniform_bytes((const unsigned char *)a.pages.v + head);
      stride = DH * 2;
      table = (const __attribute__((address_space(4))) int32_t *)uniform_bytes(a.pages.table + (size_t)b * a.pages.max_pages);
      page_bytes = ((size_t)a.Hkv << a.pages.shift) * DH * 2;
      shift = a.pages.shift;
      n_pages = a.pages.n_pages;
    } else {
      const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH * 2;
      k = uniform_bytes((const unsigned char *)a.k + first);
      v = uniform_bytes((const unsigned char *)a.v + first);
      stride = (uint32_t)a.Hkv * DH * 2;
    }
  }
  __device__ __forceinline__ void ask(int k0, int last) {  // (entries behind the last key are not looked at)
    if constexpr (PAGED) {
      ahead[0] = table[min(k0, last) >> shift];
      ahead[1] = table[min(k0 + 16, last) >> shift];
    }
  }
  // byte offsets of the two halves of the tile at k0 (asked for before)
  __device__ __forceinline__ void halves(int k0, size_t (&off)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (PAGED) {
        int page = ahead[h];
        if ((uint32_t)page >= (uint32_t)n_pages) { page = 0; bad = 1; }
        off[h] = (size_t)(uint32_t)page * page_bytes + (uint32_t)((k0 + 16 * h) & ((1 << shift) - 1)) * stride;
      } else {
        off[h] = (size_t)(k0 + 16 * h) * stride;
      }
    }
  }
};

// LDS layout of a tile of 32 keys: K rows, V rows as they lie in the cache, 16-byte chunks swapped so that the 16-byte reads of K and the
// transposing reads of V (attention_bf16.hip) cover all banks once.
template <int DH> struct KeyTile {
  static constexpr int TK = 32, ROWB = DH * 2, REGION = TK * ROWB, CH = DH / 8, RPC = 1024 / ROWB, COPIES = REGION / 1024;
  static constexpr int DB = DH / 32, KK = DH / 16;
  __device__ static __forceinline__ int k_chunk(int r, int c) { return DH == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7); }
  __device__ static __forceinline__ int v_pair(int r, int p) { return DH == 128 ? p ^ (2 * (r & 3)) : p ^ (2 * ((r >> 1) & 1)); }
  __device__ static __forceinline__ int v_chunk(int r, int c) { return (v_pair(r, c >> 1) << 1) | (c & 1); }
};

// Documents of the rows: this row's, the least and the largest of the workgroup's, and where keys of that range start and end.
// (One pass over the numbers of the sequence, 4 bytes a key, where the sweep reads 4 dh.)
__device__ __forceinline__ void doc_range(const int32_t *doc, int n, int lo, int hi, int *red, int *first, int *end) {
  int f = n, e = 0;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const int d = doc[j];
    if (d >= lo && d <= hi) {
      f = min(f, j);
      e = max(e, j + 1);
    }
  }
  f = wave_min_i(f);
  e = wave_max_i(e);
  const int w = threadIdx.x / WAVE, nw = blockDim.x / WAVE;
  if (threadIdx.x % WAVE == 0) { red[2 * w] = f; red[2 * w + 1] = e; }
  __syncthreads();
  for (int i = 0; i < nw; ++i) { f = min(f, red[2 * i]); e = max(e, red[2 * i + 1]); }
  *first = __builtin_amdgcn_readfirstlane(f);
  *end = __builtin_amdgcn_readfirstlane(e);
}

// A row's part in the masks and the scores' shape.
struct RowMask {
  int limit = 0, doc = -1;
  float pos = 0.f, slope = 0.f;  // slope in log2 units
};

// x = q.k (not scaled) -> log2 units, reshaped
struct Shape {
  float sc, cap_in, cap_out;  // scale to log2 units; 2 log2e / (sqrt(dh) cap), cap log2e
  bool capped, sloped;
  __device__ __forceinline__ Shape(const ScoredAttn &a) {
    const float scale = 1.0f / sqrtf((float)a.dh);
    sc = scale * LOG2E;
    capped = a.soft_cap > 0.f;
    sloped = a.slopes != nullptr;
    cap_in = capped ? 2.0f * LOG2E * scale / a.soft_cap : 0.f;
    cap_out = a.soft_cap * LOG2E;
  }
  // c tanh(y) = c - 2c / (1 + e^2y): an exponential and a reciprocal; both ends are right (e^2y = 0 and infinity)
  __device__ __forceinline__ float cap(float x) const {
    return fmaf(-2.0f * cap_out, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * cap_in)), cap_out);
  }
};

__device__ __forceinline__ uint32_t any_nonfinite(const uint4 &w) {  // bits 15 and 31: exponents that are all ones
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= ((&w.x)[i] & 0x7f807f80u) + 0x00800080u;
  return r;
}

// Values that are no finite numbers, in a tile where some keys count for some rows only.  A matrix product gives 0 * inf = NaN to rows that the key does
// not count for.  So these values are taken out, and what they do to rows with a weight for them is found by products with 0 and 1 (is it NaN,
// +inf, -inf) in place of the values.  Rare: no cost beyond the look at the exponents in tiles that are tested key by key.
template <int DB>
__device__ __forceinline__ void take_out_nonfinite(bf16x8 (&vf)[2][DB], const bf16x8 (&pf)[2], floatx16 (&acc)[DB]) {
  uint32_t any = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int db = 0; db < DB; ++db) any |= any_nonfinite(__builtin_bit_cast(uint4, vf[k][db]));
  if (!__any(any & 0x80008000u)) return;
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {
    const uint32_t mask = kind == 0 ? 0x7fffu : 0xffffu, base = kind == 0 ? 0x7f81u : kind == 1 ? 0x7f80u : 0xff80u, span = kind == 0 ? 0x7fu : 1u;
    const float value = __uint_as_float(kind == 0 ? 0x7fc00000u : kind == 1 ? 0x7f800000u : 0xff800000u);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      floatx16 t;
#pragma unroll
      for (int e = 0; e < 16; ++e) t[e] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 w = __builtin_bit_cast(uint4, vf[k][db]);
        uint4 is;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t u = (&w.x)[i];
          (&is.x)[i] = (((u & mask) - base) < span ? 0x3f80u : 0u) | ((((u >> 16) & mask) - base) < span ? 0x3f800000u : 0u);
        }
        t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, is), pf[k], t, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[db][e] += t[e] > 0.f ? value : 0.f;
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      uint4 w = __builtin_bit_cast(uint4, vf[k][db]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t &u = (&w.x)[i];
        if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
        if ((u & 0x7f800000u) == 0x7f800000u) u &= 0x0000ffffu;
      }
      vf[k][db] = __builtin_bit_cast(bf16x8, w);
    }
}

// Scores of a lane's 16 keys of the tile at k0 -> log2 units (SHAPED, DOCS); keys that do not count -> -inf.  Returns whether any test was
// needed (uniform).  least: the least limit of the wave's rows.  docs: the tile's 32 numbers in LDS; one: the wave's rows are of one document.
template <int MODE>
__device__ __forceinline__ bool shape_scores(floatx16 &s, const Shape &sh, const RowMask &row, int k0, int lhi, int l32, int least, const int32_t *docs, bool one) {
  const int key0 = k0 + 4 * lhi;
  if constexpr (MODE != PLAIN) {
    if (sh.capped) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = sh.cap(s[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= sh.sc;
    }
    if (sh.sloped) {
      const float d0 = row.pos - (float)key0;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = fmaf(-row.slope, fabsf(d0 - (float)(8 * (e / 4) + (e % 4))), s[e]);
    }
  }
  bool tested = false;
  if constexpr (MODE == DOCS) {
    const uint32_t same = (uint32_t)__ballot(docs[l32] == row.doc);
    if (!one) {
      tested = true;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int4 d = *reinterpret_cast<const int4 *>(docs + 4 * lhi + 8 * g);
        s[4 * g] = d.x == row.doc ? s[4 * g] : -INFINITY;
        s[4 * g + 1] = d.y == row.doc ? s[4 * g + 1] : -INFINITY;
        s[4 * g + 2] = d.z == row.doc ? s[4 * g + 2] : -INFINITY;
        s[4 * g + 3] = d.w == row.doc ? s[4 * g + 3] : -INFINITY;
      }
    } else if (same != 0xffffffffu) {
      tested = true;
      const uint32_t mine = same >> (4 * lhi);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = (mine >> (8 * (e / 4) + (e % 4))) & 1u ? s[e] : -INFINITY;
    }
  }
  if (k0 + 32 > least) {  // uniform
    tested = true;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (key0 + 8 * (e / 4) + (e % 4) >= row.limit) s[e] = -INFINITY;
  }
  return tested;
}

// un-normalised rows of a split.  (A split without a key for the row: maximum -inf, sum 0.)
template <int DH>
__device__ __forceinline__ void store_scored_partial(const ScoredAttn &a, const floatx16 (&acc_o)[DH / 32], int split, uint32_t place, int lhi, float m_run, float l_run) {
  const size_t at = (size_t)split * a.cap * a.H + place;
  float *po = a.part_o + at * DH + 4 * lhi;
#pragma unroll
  for (int db = 0; db < DH / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4 *>(po + db * 32 + 8 * g) = float4{acc_o[db][4 * g], acc_o[db][4 * g + 1], acc_o[db][4 * g + 2], acc_o[db][4 * g + 3]};
  if (lhi == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{m_run, l_run};
}

// what a row's keys sum up to -> what its values are multiplied by (a row without keys: zero)
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.0f / l; }

void launch_scored_pages_few(const ScoredAttn &a, hipStream_t s);
void launch_scored_pages_many(const ScoredAttn &a, hipStream_t s);
void launch_scored_dense_few(const ScoredAttn &a, hipStream_t s);
void launch_scored_dense_many(const ScoredAttn &a, hipStream_t s);
void launch_scored_f32(const ScoredAttn &a, hipStream_t s);

}  // namespace dy
