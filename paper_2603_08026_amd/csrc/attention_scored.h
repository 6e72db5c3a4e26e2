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

// What a kernel is made for, a bit each.  (Documents with cap or bias are one kernel, which asks for each of them as it goes; as branches of
// one kernel cap and bias cost 8 to 25 %, since every branch copies the scores.  Packed documents of 4 x 4096 tokens, 28 heads over 4 of 128: 268 us, with a
// bias 300, a cap 328, both 352: that one kernel tests every tile.)
enum ScoreMode { PLAIN = 0, CAPPED = 1, BIASED = 2, DOCS = 4, DOCS_ANY = 7 };
inline int mode_of(const ScoredAttn &a) {
  const int shape = (a.soft_cap > 0.f ? CAPPED : 0) | (a.slopes ? BIASED : 0);
  return !a.doc ? shape : shape ? DOCS_ANY : DOCS;
}

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

// Over a wave, with moves between vector registers alone, as wave_scan (a workgroup makes some ten of these before its first copy; through LDS each took 0.3 us).
template <typename T, typename Op> __device__ __forceinline__ T wave_fold(T x, Op op) {
  auto step = [&](auto ctrl_c, auto rows_c) {
    // (a lane that nothing moves to keeps its own: for minima and maxima; sums take the zero)
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const uint32_t old = Op::idempotent ? u : 0u;
    x = op(x, __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)u, decltype(ctrl_c)::value, decltype(rows_c)::value, 0xf, false)));
  };
  using every = std::integral_constant<int, 0xf>;
  step(std::integral_constant<int, 0x111>{}, every{});
  step(std::integral_constant<int, 0x112>{}, every{});
  step(std::integral_constant<int, 0x114>{}, every{});
  step(std::integral_constant<int, 0x118>{}, every{});
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_readlane((int)__builtin_bit_cast(uint32_t, x), WAVE - 1));
}
struct Least { static constexpr bool idempotent = true; __device__ int operator()(int a, int b) const { return min(a, b); } };
struct Most { static constexpr bool idempotent = true; __device__ int operator()(int a, int b) const { return max(a, b); } };
struct Sum { static constexpr bool idempotent = false; __device__ float operator()(float a, float b) const { return a + b; } };
__device__ __forceinline__ int wave_min_i(int v) { return wave_fold(v, Least{}); }
__device__ __forceinline__ int wave_max_i(int v) { return wave_fold(v, Most{}); }

// ---- work items: (key-value head, sequence, key split, tile of packed rows) ---------------------------------------
// The rows of a sequence and the g heads of a group are packed as in the grouped form above.  Where rows are few the keys of a sequence are split, in
// pieces of one size for all sequences, the smallest with which no more than a.target items are made: workgroups of ragged requests then
// end together, and fit the chip in one round.  (The lengths are the device's to know.)
constexpr int SPLIT_KEYS = 128;  // keys that the waves of a workgroup take at a time; a split has a multiple
inline long scored_tiles(const ScoredAttn &a) {  // at most, of one key-value head
  const long g = a.H / a.Hkv;
  return a.offsets ? (a.cap * g + a.bq - 1) / a.bq + a.B : a.B * ((a.L * g + a.bq - 1) / a.bq);
}
inline long scored_items(const ScoredAttn &a) {
  return scored_tiles(a) + (a.splits > 1 ? (a.target + a.Hkv - 1) / a.Hkv : 0);  // (where the sizes of the pieces were not found: sum of ceilings)
}
// Which of the 8 XCDs takes which item: the tiles that read one (sequence, head)'s keys stay on as few as the heads allow, next to each other in time.
inline long scored_grid(const ScoredAttn &a) {
  const long t = scored_items(a);
  return (t * a.Hkv + ATTN_XCD - 1) / ATTN_XCD * ATTN_XCD;
}
struct ScoredItem {
  int seq = -1, row = 0, packed = 0, n = 0;  // as AttnItem
  int kv_head = 0, keys = 0, split = 0, splits = 1, chunk = 0;
  int counter = 0;  // number of the (tile, key-value head)
};
struct ScoredSeq { int lo = 0, rows = 0, tiles = 0, keys = 0; };
__device__ __forceinline__ int scored_rows(const ScoredAttn &a) { return a.offsets ? max(min(a.offsets[a.B], a.cap), 0) : a.B * a.L; }
__device__ __forceinline__ ScoredSeq scored_seq(const ScoredAttn &a, int b, int total) {
  ScoredSeq q;
  if (b >= a.B) return q;
  q.lo = a.offsets ? min(max(a.offsets[b], 0), total) : b * a.L;
  q.rows = a.offsets ? max(min(a.offsets[b + 1], total), q.lo) - q.lo : a.L;
  q.tiles = (q.rows * (a.H / a.Hkv) + a.bq - 1) / a.bq;
  q.keys = keys_of(a, b);
  return q;
}
// keys of a split of a sequence (no more than a.splits of them), and how many splits that makes
__device__ __forceinline__ int split_size(const ScoredAttn &a, int keys, int chunk) {
  return max(chunk, ((keys + a.splits - 1) / a.splits + SPLIT_KEYS - 1) / SPLIT_KEYS * SPLIT_KEYS);
}
__device__ __forceinline__ int split_count(int keys, int size) { return max(1, (int)(((long)keys + size - 1) / size)); }
constexpr int WHOLE = 0x7fffff80;  // a piece that holds any sequence
// A first size from the sum of tiles * keys, then what it makes of the sequences' ends.  sum: (function of a sequence -> number) -> its sum over all of
// them; sums of whole numbers in a fixed order, every workgroup finds the same.
template <typename SUM> __device__ __forceinline__ int scored_chunk(const ScoredAttn &a, SUM &&sum) {
  if (a.splits <= 1) return WHOLE;
  int chunk = WHOLE;
  float pieces = sum([&](const ScoredSeq &q) { return (float)q.tiles * (float)q.keys; }) * (float)a.Hkv / (float)a.target;
#pragma unroll 1
  for (int round = 0; round < 4; ++round) {
    chunk = max((int)ceilf(fminf(pieces, 1e9f) / SPLIT_KEYS), 1) * SPLIT_KEYS;
    const float items = sum([&](const ScoredSeq &q) { return (float)(q.tiles * split_count(q.keys, split_size(a, q.keys, chunk))); }) * (float)a.Hkv;
    if (items <= (float)a.target) break;  // uniform
    pieces = (float)chunk * fmaxf(items / (float)a.target, 1.02f);
  }
  return chunk;
}
// item p of the grid -> key-value head and item of that head, of n_items
__device__ __forceinline__ bool scored_place(const ScoredAttn &a, int p, int n_items, int *kv_head, int *w) {
  if (n_items == 0) return false;
  const int x = p % ATTN_XCD, s = p / ATTN_XCD;
  if (a.Hkv % ATTN_XCD == 0) {
    const int per = a.Hkv / ATTN_XCD;
    *kv_head = x * per + s / n_items;
    *w = s % n_items;
    return s / n_items < per;
  }
  if (ATTN_XCD % a.Hkv == 0) {
    const int per = ATTN_XCD / a.Hkv;
    *kv_head = x / per;
    *w = s * per + x % per;
    return *w < n_items;
  }
  const long items = (long)n_items * a.Hkv, per_xcd = (items + ATTN_XCD - 1) / ATTN_XCD, at = x * per_xcd + s;
  *kv_head = (int)(at / n_items);
  *w = (int)(at % n_items);
  return s < per_xcd && at < items;
}
// mine: item of the sequence; tiles_before: tiles of the sequences before it
__device__ __forceinline__ void scored_fill(const ScoredAttn &a, ScoredItem &it, const ScoredSeq &q, int chunk, int mine, int tiles_before, int n_tiles) {
  it.row = q.lo;
  it.keys = q.keys;
  it.chunk = split_size(a, q.keys, chunk);
  it.splits = split_count(q.keys, it.chunk);
  it.split = mine / q.tiles;
  const int tile = q.tiles - 1 - mine % q.tiles;  // the last rows of a causal sequence have the most keys: they come first
  it.counter = it.kv_head * n_tiles + tiles_before + tile;  // (below ARRIVE_WORDS where there are splits: scored_plan)
  it.packed = tile * a.bq;
  it.n = min(a.bq, q.rows * (a.H / a.Hkv) - it.packed);
}
// Offsets that descend name some rows twice: that would be more tiles than the grid and the counters were made for, and a counter that never comes to its
// end stays for later calls.  So a call with such offsets has no items at all, and says so in the status word.
__device__ __forceinline__ bool descends(const ScoredAttn &a, int b) { return a.offsets && b < a.B && a.offsets[b + 1] < a.offsets[b]; }
// Up to 64 sequences: every workgroup looks at all of them, a lane at one.  More: k_scored_list has left, for every sequence, the items and tiles of it and
// those before it, and the size of the pieces; a search over 64 equal parts, then inside one.
constexpr int LIST_HEAD = 1;  // words before the two lists: the size of the pieces, 0 where offsets descend
__device__ __forceinline__ bool no_order(const ScoredAttn &a) {  // uniform
  return a.B <= WAVE ? __any(descends(a, threadIdx.x % WAVE)) : a.list[0] == 0;
}
__device__ __forceinline__ ScoredItem scored_item(const ScoredAttn &a, int p) {
  const int lane = threadIdx.x % WAVE, total = scored_rows(a);
  ScoredItem it;
  int w;
  if (a.B <= WAVE) {
    const ScoredSeq q = scored_seq(a, lane, total);
    const bool down = no_order(a);
    const int chunk = scored_chunk(a, [&](auto f) { return wave_fold(f(q), Sum{}); });
    const int upto = wave_scan(q.tiles * split_count(q.keys, split_size(a, q.keys, chunk))), tiles_to = wave_scan(q.tiles);
    if (!scored_place(a, p, down ? 0 : __builtin_amdgcn_readlane(upto, WAVE - 1), &it.kv_head, &w)) {
      if (down) *a.status = a.bad_offsets_code;  // (all threads: with one picked out the documents' kernel spills 26 registers in place of 9, 269 -> 277 us)
      return it;
    }
    const int f = __ffsll((unsigned long long)__ballot(upto > w)) - 1;
    const int before = f ? __builtin_amdgcn_readlane(upto, f - 1) : 0, tiles_before = f ? __builtin_amdgcn_readlane(tiles_to, f - 1) : 0;
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, f); };
    it.seq = f;
    scored_fill(a, it, ScoredSeq{of(q.lo), of(q.rows), of(q.tiles), of(q.keys)}, chunk, w - before, tiles_before, __builtin_amdgcn_readlane(tiles_to, WAVE - 1));
    return it;
  }
  const int32_t *items_to = a.list + LIST_HEAD, *tiles_to = items_to + a.B;
  const int step = (a.B + WAVE - 1) / WAVE, chunk = a.list[0], n_tiles = tiles_to[a.B - 1];
  const int part_end = items_to[min((lane + 1) * step, a.B) - 1];
  if (!scored_place(a, p, __builtin_amdgcn_readlane(part_end, WAVE - 1), &it.kv_head, &w)) return it;
  const int part = __ffsll((unsigned long long)__ballot(part_end > w)) - 1;
  for (int r0 = part * step; it.seq < 0; r0 += WAVE) {  // (the part's end is past w, so one is found)
    if (r0 >= a.B) return it;
    const uint64_t past = __ballot(items_to[min(r0 + lane, a.B - 1)] > w);
    if (past) it.seq = __builtin_amdgcn_readfirstlane(r0 + __ffsll((unsigned long long)past) - 1);
  }
  const ScoredSeq q = scored_seq(a, it.seq, total);
  scored_fill(a, it, q, chunk, w - (it.seq ? items_to[it.seq - 1] : 0), it.seq ? tiles_to[it.seq - 1] : 0, n_tiles);
  return it;
}

// ---- key splits: partial results, and their merge ------------------------------------------------------------------------
// Few rows (a.fused): by the workgroup that arrives last.  Partial rows, their maxima (log2 units) and sums go past the caches of the die (device
// scope), so that workgroups on other dies see them without a flush: stored, waited for, then counted.  The one that finds all others of its (tile,
// head) counted merges, and leaves the counter at zero.  Many rows: by a launch of its own (k_scored_merge), which has the whole chip for them.
// One token of one request of 32768 keys, 28 heads over 4: launch of its own / last one 44 / 28 us; of 8 requests of 8192, 8 over 2 of 64, 21.7 / 18.4; but 32 rows
// of 16 x 1280 keys, 32 heads, 92 / 121.
constexpr int MAX_SPLITS = 128;
__device__ __forceinline__ void store_through(float *p, float2 v) {
  __hip_atomic_store(reinterpret_cast<uint64_t *>(p), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_through(const float *p) {
  return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// what a row's keys sum up to -> what its values are multiplied by (a row without keys: zero)
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.0f / l; }

// Called by all 256 threads, whose partial results are stored (not waited for).  flag: a word of LDS; buf: 4 * DH floats of it.
// Eight rows at a time (a tile has more where one sequence has most of the rows); a row is taken by four waves, by two or by one, a wave takes up to
// two of the eight: 16 splits of each are in flight.
constexpr int FUSED_ROWS = 8;
template <typename T, int DH> __device__ __forceinline__ void merge_splits_last(const ScoredAttn &a, const ScoredItem &item, int *flag, float *buf) {
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), grp = a.H / a.Hkv, splits = item.splits;
  wait_vmcnt<0>();
  __syncthreads();
  if (tid == 0) {
    const int before = __hip_atomic_fetch_add(a.arrive + item.counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == splits - 1) __hip_atomic_store(a.arrive + item.counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = before == splits - 1;
  }
  __syncthreads();
  if (!*flag) return;
  constexpr int V = DH / WAVE, IN_FLIGHT = 16;
  auto load = [&](const float *p, float (&x)[V]) {
    if constexpr (V == 2) {
      const float2 v = load_through(p);
      x[0] = v.x; x[1] = v.y;
    } else {
      x[0] = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  };
  const int parts = item.n == 1 ? 4 : item.n == 2 ? 2 : 1, part = wave % parts;  // waves of a row
  const size_t step = (size_t)a.cap * a.H;
  for (int first = wave / parts; first < item.n; first += FUSED_ROWS) {  // (once where waves share rows)
    const bool second = first + 4 < item.n;
    size_t at[2];
    float m[2][2], l[2][2], o[2][V], total[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int p = item.packed + (u && second ? first + 4 : first);
      at[u] = (size_t)(item.row + p / grp) * a.H + item.kv_head * grp + p % grp;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int s = lane + h * WAVE;
        const float2 ml = s < splits ? load_through(a.part_ml + (s * step + at[u]) * 2) : float2{-INFINITY, 0.f};
        m[u][h] = ml.x; l[u][h] = ml.y;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) o[u][e] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // m becomes the weights
      const float M = wave_max(fmaxf(m[u][0], m[u][1])), ref = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int h = 0; h < 2; ++h) m[u][h] = __builtin_amdgcn_exp2f(m[u][h] - ref);
      total[u] = wave_sum(l[u][0] * m[u][0] + l[u][1] * m[u][1]);
    }
    auto rows = [&](auto count_c) {
      constexpr int N = decltype(count_c)::value;
      for (int s0 = part; s0 < splits; s0 += IN_FLIGHT * parts) {  // (past the end the last split again, with no weight)
        float x[N][IN_FLIGHT][V];
#pragma unroll
        for (int i = 0; i < IN_FLIGHT; ++i)
#pragma unroll
          for (int u = 0; u < N; ++u) load(a.part_o + (min(s0 + i * parts, splits - 1) * step + at[u]) * DH + lane * V, x[u][i]);
#pragma unroll
        for (int i = 0; i < IN_FLIGHT; ++i) {
          const int s = s0 + i * parts;
          if (s >= splits) break;  // uniform
#pragma unroll
          for (int u = 0; u < N; ++u) {
            const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s < WAVE ? m[u][0] : m[u][1]), s % WAVE));
#pragma unroll
            for (int e = 0; e < V; ++e) o[u][e] = fmaf(x[u][i][e], w, o[u][e]);
          }
        }
      }
    };
    if (second) rows(std::integral_constant<int, 2>{});
    else rows(std::integral_constant<int, 1>{});
    if (parts > 1) {
#pragma unroll
      for (int e = 0; e < V; ++e) buf[(wave * V + e) * WAVE + lane] = o[0][e];
      __syncthreads();
      if (part > 0) return;
      for (int w = 1; w < parts; ++w)
#pragma unroll
        for (int e = 0; e < V; ++e) o[0][e] += buf[((wave + w) * V + e) * WAVE + lane];
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u && !second) break;
      const float inv = inverse_of(total[u]);
#pragma unroll
      for (int e = 0; e < V; ++e) ((T *)a.out)[at[u] * DH + lane * V + e] = from_f<T>(o[u][e] * inv);
    }
  }
}

// ---- shared pieces of the bf16 kernels -----------------------------------------------------------------------
__device__ __forceinline__ const unsigned char *uniform_bytes(const void *p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (const unsigned char *)(((uint64_t)hi << 32) | lo);
}
// Where the keys and values of a sequence and head lie.  A tile of 32 keys starts at a multiple of 32, pages hold a multiple of 16: its two halves
// lie each in one piece.  PAGED: their pages are asked for through the scalar cache, a tile ahead.
template <bool PAGED, int DH, int BYTES = 2> struct KeyPlaces {  // BYTES of an element
  const unsigned char *k, *v;             // of key 0 (pages: of page 0)
  uint32_t stride;                        // bytes from one key to the next
  const __attribute__((address_space(4))) int32_t *table;
  size_t page_bytes;
  int shift, n_pages, bad = 0;
  int ahead[2];                           // pages of the tile asked for
  __device__ __forceinline__ KeyPlaces(const ScoredAttn &a, int b, int kvh) {
    if constexpr (PAGED) {
      const size_t head = ((size_t)kvh << a.pages.shift) * DH * BYTES;
      k = uniform_bytes((const unsigned char *)a.pages.k + head);
      v = uniform_bytes((const unsigned char *)a.pages.v + head);
      stride = DH * BYTES;
      table = (const __attribute__((address_space(4))) int32_t *)uniform_bytes(a.pages.table + (size_t)b * a.pages.max_pages);
      page_bytes = ((size_t)a.Hkv << a.pages.shift) * DH * BYTES;
      shift = a.pages.shift;
      n_pages = a.pages.n_pages;
    } else {
      const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH * BYTES;
      k = uniform_bytes((const unsigned char *)a.k + first);
      v = uniform_bytes((const unsigned char *)a.v + first);
      stride = (uint32_t)a.Hkv * DH * BYTES;
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

// Where keys of documents from lo to hi, those of a workgroup's rows, start and end, and whether all keys in between are of the one document that the rows
// are of.  (One pass over the numbers of the sequence, 4 bytes a key, where the sweep reads 4 dh.)  red: 12 words of LDS.
__device__ __forceinline__ void doc_range(const int32_t *doc, int n, int lo, int hi, int *red, int *first, int *end, bool *solid) {
  int f = n, e = 0, count = 0;
  constexpr int U = 8;  // numbers a thread has in flight
  for (int j0 = threadIdx.x; j0 < n; j0 += 256 * U) {
    int d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) d[u] = doc[min(j0 + 256 * u, n - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + 256 * u;
      if (j < n && d[u] >= lo && d[u] <= hi) {
        f = min(f, j);
        e = max(e, j + 1);
        ++count;
      }
    }
  }
  f = wave_min_i(f);
  e = wave_max_i(e);
  count = __builtin_amdgcn_readlane(wave_scan(count), WAVE - 1);
  const int w = threadIdx.x / WAVE;
  if (threadIdx.x % WAVE == 0) { red[3 * w] = f; red[3 * w + 1] = e; red[3 * w + 2] = count; }
  __syncthreads();
  count = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f = min(f, red[3 * i]);
    e = max(e, red[3 * i + 1]);
    count += red[3 * i + 2];
  }
  *first = __builtin_amdgcn_readfirstlane(f);
  *end = __builtin_amdgcn_readfirstlane(e);
  *solid = lo == hi && __builtin_amdgcn_readfirstlane(count) == *end - *first;
}

// A row's part in the masks and the scores' shape.
struct RowMask {
  int limit = 0, doc = -1;
  int pos = 0;        // (distances are taken between whole numbers: positions may exceed 2^24)
  float slope = 0.f;  // slope in units of the score as it goes into the exponential's multiply-add
};

// x = q.k (not scaled) -> reshaped; x * sc is in log2 units (a capped one is so itself: sc = 1)
struct Shape {
  float sc, cap_in, cap_out;  // cap_in = 2 log2e / (sqrt(dh) cap), cap_out = cap log2e
  bool capped, sloped;
  __device__ __forceinline__ Shape(const ScoredAttn &a) {
    const float scale = 1.0f / sqrtf((float)a.dh);
    capped = a.soft_cap > 0.f;
    sloped = a.slopes != nullptr;
    sc = capped ? 1.f : scale * LOG2E;
    cap_in = capped ? 2.0f * LOG2E * scale / a.soft_cap : 0.f;
    cap_out = a.soft_cap * LOG2E;
  }
  __device__ __forceinline__ float slope(float x) const { return x * LOG2E / sc; }
  // c tanh(y) = c - 2c / (1 + e^2y): an exponential and a reciprocal; both ends are right (e^2y = 0 and infinity)
  __device__ __forceinline__ float cap(float x) const {
    return fmaf(-2.0f * cap_out, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * cap_in)), cap_out);
  }
};

// fp32: tanh by itself, as exact for small scores as for large ones (the difference of two numbers of the cap's size loses what a score is smaller: 4.9e-4 of
// a score of 1 at a cap of 4096).  200 rows of each of 16 sequences of 2048 keys, 16 heads over 4 of 128: no cap 598 us, a cap 682, by the difference 623.
struct ShapeF32 : Shape {
  float cap_by;  // 1 / (sqrt(dh) cap)
  __device__ __forceinline__ ShapeF32(const ScoredAttn &a) : Shape(a) { cap_by = capped ? 1.0f / sqrtf((float)a.dh) / a.soft_cap : 0.f; }
  __device__ __forceinline__ float cap(float x) const { return cap_out * tanhf(x * cap_by); }
};

// Values that are no finite numbers, in a tile where some keys count for some rows only.  A matrix product gives 0 * inf = NaN to rows that the key does
// not count for.  So these values are taken out, and what they do to rows with a weight for them is found by products with 0 and 1 (is it NaN,
// +inf, -inf) in place of the values.  Rare: no cost beyond the look at the values of tiles that are tested key by key.
template <int DB>
__device__ __forceinline__ void take_out_nonfinite(bf16x8 (&vf)[2][DB], const bf16x8 (&pf)[2], floatx16 (&acc)[DB]) {
  float none = 0.f;  // 0 times a number is 0, times anything else NaN: two values an instruction
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const uint4 w = __builtin_bit_cast(uint4, vf[k][db]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t u = (&w.x)[i];
        none = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, u), __builtin_bit_cast(bf16x2_t, 0u), none, false);
      }
    }
  if (!__any(none != 0.f)) return;
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

// What a tile's keys have to be tested for.
struct TileTests {
  int least = 0;       // limits of the wave's rows: the least
  int first = 0;       // documents: keys below do not count
  bool one = true;     // ... the wave's rows are of one
  bool solid = false;  // ... and so are all keys from `first` to the largest limit
};
// Scores of a lane's 16 keys of the tile at k0, reshaped; keys that do not count -> -inf.  Returns whether any was tested (uniform).  docs: the tile's
// 32 numbers in LDS.
template <int MODE, typename SHAPE>
__device__ __forceinline__ bool shape_scores(floatx16 &s, const SHAPE &sh, const RowMask &row, const TileTests &t, int k0, int lhi, int l32, const int32_t *docs) {
  const int key0 = k0 + 4 * lhi;
  if constexpr (MODE & CAPPED) {
    if (MODE != DOCS_ANY || sh.capped) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = sh.cap(s[e]);
    }
  }
  if constexpr (MODE & BIASED) {
    if (MODE != DOCS_ANY || sh.sloped) {
      const float d0 = (float)(row.pos - key0);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = fmaf(-row.slope, fabsf(d0 - (float)(8 * (e / 4) + (e % 4))), s[e]);
    }
  }
  bool tested = false;
  if constexpr (MODE & DOCS) {
    if (t.solid) {
      if (k0 < t.first) {  // uniform
        tested = true;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (key0 + 8 * (e / 4) + (e % 4) < t.first) s[e] = -INFINITY;
      }
    } else if (!t.one) {
      tested = true;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int4 d = *reinterpret_cast<const int4 *>(docs + 4 * lhi + 8 * g);
        s[4 * g] = d.x == row.doc ? s[4 * g] : -INFINITY;
        s[4 * g + 1] = d.y == row.doc ? s[4 * g + 1] : -INFINITY;
        s[4 * g + 2] = d.z == row.doc ? s[4 * g + 2] : -INFINITY;
        s[4 * g + 3] = d.w == row.doc ? s[4 * g + 3] : -INFINITY;
      }
    } else if (const uint32_t same = (uint32_t)__ballot(docs[l32] == row.doc); same != 0xffffffffu) {
      tested = true;
      const uint32_t mine = same >> (4 * lhi);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = (mine >> (8 * (e / 4) + (e % 4))) & 1u ? s[e] : -INFINITY;
    }
  }
  if (k0 + 32 > t.least) {  // uniform
    tested = true;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (key0 + 8 * (e / 4) + (e % 4) >= row.limit) s[e] = -INFINITY;
  }
  return tested;
}

// un-normalised rows of a split.  (A split without a key for the row: maximum -inf, sum 0.)
template <int DH>
__device__ __forceinline__ void store_scored_partial(const ScoredAttn &a, const floatx16 (&acc_o)[DH / 32], const ScoredItem &item, uint32_t place, int jq, int lhi, float m_run, float l_run) {
  const size_t at = (size_t)item.split * a.cap * a.H + place;
  float *po = a.part_o + at * DH + 4 * lhi;
  if (a.fused) {
#pragma unroll
    for (int db = 0; db < DH / 32; ++db)
#pragma unroll
      for (int g = 0; g < 8; ++g) store_through(po + db * 32 + 8 * (g / 2) + 2 * (g % 2), float2{acc_o[db][2 * g], acc_o[db][2 * g + 1]});
    if (lhi == 0) store_through(a.part_ml + at * 2, float2{m_run, l_run});
    return;
  }
#pragma unroll
  for (int db = 0; db < DH / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4 *>(po + db * 32 + 8 * g) = float4{acc_o[db][4 * g], acc_o[db][4 * g + 1], acc_o[db][4 * g + 2], acc_o[db][4 * g + 3]};
  if (lhi == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{m_run, l_run};
}

// (a.once: keys and values past the L2)
void launch_scored_pages_few(const ScoredAttn &a, hipStream_t s);
void launch_scored_pages_many(const ScoredAttn &a, hipStream_t s);
void launch_scored_pages_once(const ScoredAttn &a, hipStream_t s);
void launch_scored_dense_few(const ScoredAttn &a, hipStream_t s);
void launch_scored_dense_many(const ScoredAttn &a, hipStream_t s);
void launch_scored_dense_once(const ScoredAttn &a, hipStream_t s);

}  // namespace dy
