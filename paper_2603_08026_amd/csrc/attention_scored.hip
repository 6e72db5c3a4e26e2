// Attention with masked and reshaped scores: fp32, and which kernel takes a call.
#include "attention_scored.h"
#include <float.h>
#include <math.h>
#include <algorithm>

namespace dy {

namespace {

// ---- fp32: R packed rows a workgroup -------------------------------------------------------------------------------
// dh / 16 lanes take a key, a lane 16 of its elements, and 64 / (dh / 16) keys go through a wave at a time, each group of lanes with a running
// maximum, sum and result of its own; four waves take such steps in turn, and groups and waves are merged at the end.  K and V go straight into
// registers, a step ahead, the pages' numbers another.  Every product and sum is fp32.  Bound by the latency of few steps, then by the vector ALU and by
// reading K and V from the L2 for every two rows: one token of each of 16 requests of 2048 keys, 4 heads of 64, 19.8 us, 3.4 TB/s.  (Many rows: the tile below.)
template <int DH, bool PAGED, int R>
__global__ __launch_bounds__(256, 2) void k_scored_f32(ScoredAttn a) {
  constexpr int EPL = 16, LPK = DH / EPL, KS = WAVE / LPK, NW = 4;  // elements of a lane, lanes of a key, keys of a step
  __shared__ float part[NW][R][DH], part_ml[NW][R][2];
  __shared__ float buf[4 * DH];
  __shared__ int red[3 * NW];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int c = lane % LPK, group = lane / LPK;
  const ScoredItem item = scored_item(a, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such item
  const int nq = item.n, grp = a.H / a.Hkv;
  auto row_of = [&](int r) { return item.row + (item.packed + r) / grp; };
  auto head_of = [&](int r) { return kvh * grp + (item.packed + r) % grp; };
  auto place = [&](int r) { return (uint32_t)row_of(r) * (uint32_t)a.H + (uint32_t)head_of(r); };
  RowMask row[R];
  int k_lo = split * item.chunk, k_hi = 0, lo = 0x7fffffff, hi = -1, least = 0x7fffffff;
  const int32_t *docs = a.doc ? a.doc + (size_t)b * a.L : nullptr;
#pragma unroll
  for (int r = 0; r < R; ++r) {  // (rows past the end: the last one again, their results are never stored)
    const int rr = min(r, nq - 1), i = position_of(a, PAGED, b, row_of(rr));
    row[r].limit = limit_of(a, b, item.keys, i);
    row[r].pos = i;
    row[r].slope = a.slopes ? a.slopes[head_of(rr)] * LOG2E : 0.f;  // (scores are kept in the log2 domain)
    if (docs) {
      row[r].doc = i >= 0 && i < a.L ? docs[i] : -1;
      if (row[r].doc < 0) row[r].limit = 0;
      lo = min(lo, row[r].doc < 0 ? 0x7fffffff : row[r].doc);
      hi = max(hi, row[r].doc);
    }
    k_hi = max(k_hi, row[r].limit);
    least = min(least, row[r].limit);
  }
  k_hi = min(k_hi, (int)min((long)k_lo + item.chunk, 0x7fffffffl));
  if (docs) {
    int first, end;
    bool solid;
    doc_range(docs, item.keys, lo, hi, red, &first, &end, &solid);
    k_hi = min(k_hi, end);
    k_lo = max(k_lo, first);
  }
  const Shape sh(a);
  float q[R][EPL], acc[R][EPL], m_run[R], l_run[R];
  const float scale = 1.0f / sqrtf((float)DH), by = sh.capped ? scale / a.soft_cap : scale * LOG2E;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float4 *src = reinterpret_cast<const float4 *>((const float *)a.q + (size_t)place(min(r, nq - 1)) * DH + c * EPL);
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) {
      const float4 x = src[i];
      q[r][4 * i] = x.x * by; q[r][4 * i + 1] = x.y * by; q[r][4 * i + 2] = x.z * by; q[r][4 * i + 3] = x.w * by;
    }
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[r][e] = 0.f;
    m_run[r] = -FLT_MAX;  // (finite, so that a score of -inf has the probability 0)
    l_run[r] = 0.f;
  }
  const size_t dense = ((size_t)b * a.L * a.Hkv + kvh) * DH + c * EPL, head = ((size_t)kvh << a.pages.shift) * DH + c * EPL;
  const int32_t *table = PAGED ? a.pages.table + (size_t)b * a.pages.max_pages : nullptr;
  const float *kp = (const float *)(PAGED ? a.pages.k : a.k) + (PAGED ? head : dense), *vp = (const float *)(PAGED ? a.pages.v : a.v) + (PAGED ? head : dense);
  bool bad = false;
  struct Step { float k[EPL], v[EPL]; int doc; };
  auto key_of = [&](int n) { return k_lo + (n * NW + wave) * KS + group; };
  auto page_of = [&](int n) { return PAGED ? table[min(key_of(n), k_hi - 1) >> a.pages.shift] : 0; };  // (keys past the end: the last one again, masked later)
  auto load = [&](int n, int page, Step &s) {
    const int key = min(key_of(n), k_hi - 1);
    size_t at;
    if constexpr (PAGED) {
      if ((uint32_t)page >= (uint32_t)a.pages.n_pages) { page = 0; bad = true; }
      at = ((((size_t)(uint32_t)page * a.Hkv) << a.pages.shift) + (uint32_t)(key & ((1 << a.pages.shift) - 1))) * DH;
    } else {
      at = (size_t)key * a.Hkv * DH;
    }
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) {
      const float4 x = reinterpret_cast<const float4 *>(kp + at)[i], y = reinterpret_cast<const float4 *>(vp + at)[i];
      s.k[4 * i] = x.x; s.k[4 * i + 1] = x.y; s.k[4 * i + 2] = x.z; s.k[4 * i + 3] = x.w;
      s.v[4 * i] = y.x; s.v[4 * i + 1] = y.y; s.v[4 * i + 2] = y.z; s.v[4 * i + 3] = y.w;
    }
    s.doc = docs ? docs[key] : 0;
  };
  const int n_steps = k_hi > k_lo ? (k_hi - k_lo + NW * KS - 1) / (NW * KS) : 0;
  Step next;
  int page = 0;
  if (n_steps > 0) {
    load(0, page_of(0), next);
    page = page_of(1);
  }
  for (int n = 0; n < n_steps; ++n) {
    const Step now = next;
    if (n + 1 < n_steps) {
      load(n + 1, page, next);
      page = page_of(n + 2);
    }
    float score[R];
    bool need = false;
    const int key = key_of(n);
    const bool tested = docs || k_lo + (n + 1) * NW * KS > min(k_hi, least);  // uniform
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float d0 = 0.f, d1 = 0.f;
#pragma unroll
      for (int e = 0; e < EPL; e += 2) {
        d0 = fmaf(q[r][e], now.k[e], d0);
        d1 = fmaf(q[r][e + 1], now.k[e + 1], d1);
      }
      float x = lanes_sum<LPK>(d0 + d1);
      if (sh.capped) x = sh.cap_out * tanhf(x);
      if (sh.sloped) x = fmaf(-row[r].slope, fabsf((float)(row[r].pos - key)), x);
      if (tested) x = key < k_hi && key < row[r].limit && (!docs || now.doc == row[r].doc) ? x : -INFINITY;
      score[r] = x;
      need = need || x > m_run[r] + 8.0f;
    }
    if (__any(need)) {  // the running reference moves where a score exceeds it by more than 2^8: rare after the first steps
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float top = fmaxf(m_run[r], score[r]);
        const float corr = __builtin_amdgcn_exp2f(m_run[r] - top);
        m_run[r] = top;
        l_run[r] *= corr;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[r][e] *= corr;
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (tested) {  // (a value that does not count may be no number)
        const bool counts = score[r] != -INFINITY;
        const float p = counts ? __builtin_amdgcn_exp2f(score[r] - m_run[r]) : 0.f;
        l_run[r] += p;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[r][e] = fmaf(p, counts ? now.v[e] : 0.f, acc[r][e]);
      } else {
        const float p = __builtin_amdgcn_exp2f(score[r] - m_run[r]);
        l_run[r] += p;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[r][e] = fmaf(p, now.v[e], acc[r][e]);
      }
    }
  }
  if (PAGED && bad) *a.status = a.bad_page_code;
  // merge of a wave's groups: each exchange halves the elements that a lane answers for
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float top = m_run[r];
#pragma unroll
    for (int off = LPK; off < WAVE; off *= 2) top = fmaxf(top, __shfl_xor(top, off, WAVE));
    const float w = __builtin_amdgcn_exp2f(m_run[r] - top);
    float l = l_run[r] * w;
#pragma unroll
    for (int off = LPK; off < WAVE; off *= 2) l += __shfl_xor(l, off, WAVE);
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[r][e] *= w;
    int col = c * EPL;
#pragma unroll
    for (int off = WAVE / 2, half = EPL / 2; off >= LPK; off /= 2, half /= 2) {
      const bool up = lane & off;
#pragma unroll
      for (int e = 0; e < half; ++e) {
        const float keep = up ? acc[r][e + half] : acc[r][e], send = up ? acc[r][e] : acc[r][e + half];
        acc[r][e] = keep + __shfl_xor(send, off, WAVE);
      }
      col += up ? half : 0;
    }
#pragma unroll
    for (int e = 0; e < EPL / KS; ++e) part[wave][r][col + e] = acc[r][e];
    if (lane == 0) {
      part_ml[wave][r][0] = top;
      part_ml[wave][r][1] = l;
    }
  }
  __syncthreads();
  // merge of the waves
  const bool whole = item.splits == 1;
  for (int i = tid; i < nq * DH / 2; i += 256) {
    const int r = i / (DH / 2), col = 2 * (i % (DH / 2));
    float top = part_ml[0][r][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, part_ml[w][r][0]);
    float2 o{0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(part_ml[w][r][0] - top);
      o.x = fmaf(part[w][r][col], f, o.x);
      o.y = fmaf(part[w][r][col + 1], f, o.y);
      l = fmaf(part_ml[w][r][1], f, l);
    }
    if (whole) {
      const float inv = inverse_of(l);
      *reinterpret_cast<float2 *>((float *)a.out + (size_t)place(r) * DH + col) = float2{o.x * inv, o.y * inv};
    } else {  // (a split without keys counts for nothing)
      const size_t at = (size_t)split * a.cap * a.H + place(r);
      store_through(a.part_o + at * DH + col, o);
      if (col == 0) store_through(a.part_ml + at * 2, float2{l == 0.f ? -INFINITY : top, l});
    }
  }
  if (!whole) merge_splits_last<float, DH>(a, item, red, buf);
}

// ---- fp32: 32 packed rows a workgroup ------------------------------------------------------------------------------
// S^T = K Q^T and O^T = V^T P^T by the fp32 matrix instruction, 2 keys or columns deep: a wave's lower lanes give one of the two, its upper ones the
// other, in any order that both operands share.  So K and Q split their columns in halves (a lane reads one key's half, 16 bytes at a time), and a
// product over keys takes those 4 apart that the scores' layout has in one register of either half: P^T needs no move, V comes as rows lie (a lane
// has neighbouring columns), and no operand passes through LDS.  Waves take tiles of 32 keys in turn, each with a running maximum, sum and result of
// its own; V of a tile is on its way during the scores, K of the next one during the product with V.
// Bound by the matrix pipe (2 x 2 dh x 32 x 32 operations a tile at 256 a cycle and CU) and the loads' addresses, a line a lane for K.  200 rows of each of
// 16 requests of 2048 keys, 16 heads over 4 of 128: 597 us, 90 TFLOP/s (two rows a workgroup: 2955); 8 heads over 2 of 64 176 / 797; 32 rows of each
// of 4 of 512, 4 heads of 64, 17.4 / 13.5.  (71 to 143 scalar registers go to lanes of vector registers, none to memory.)
template <int DH, bool PAGED>
__global__ __launch_bounds__(256, DH == 64 ? 2 : 1) void k_scored_f32_tile(ScoredAttn a) {
  constexpr int TK = 32, DB = DH / 32, HALF = DH / 2, NW = 4, PER_WAVE = (DB * 16 + 2) * 64;
  __shared__ __align__(16) float mg[(NW - 1) * PER_WAVE];
  __shared__ __align__(16) int32_t docs[NW][TK];
  __shared__ int red[3 * NW];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int l32 = lane % 32, lhi = lane / 32;
  const ScoredItem item = scored_item(a, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such item
  const int nq = item.n, grp = a.H / a.Hkv;
  // this lane's query (rows past the end: the last one again, their results are never stored)
  const int p = item.packed + min(l32, nq - 1), jq = item.row + p / grp, hq = kvh * grp + p % grp;
  const uint32_t place = (uint32_t)jq * (uint32_t)a.H + (uint32_t)hq;
  const ShapeF32 sh(a);
  RowMask row;
  TileTests tests;
  int k_lo = split * item.chunk;
  const int i = position_of(a, PAGED, b, jq);
  row.limit = limit_of(a, b, item.keys, i);
  row.pos = i;
  if (a.slopes) row.slope = sh.slope(a.slopes[hq]);
  const int32_t *doc = !PAGED && a.doc ? a.doc + (size_t)b * a.L : nullptr;
  if (doc) {
    row.doc = i >= 0 && i < a.L ? doc[i] : -1;
    if (row.doc < 0) row.limit = 0;
    const int some = row.doc < 0 ? 0x7fffffff : row.doc, lo = wave_min_i(some), hi = wave_max_i(row.doc);
    tests.one = __all(row.doc == hi);
    int end;
    doc_range(doc, item.keys, lo, hi, red, &tests.first, &end, &tests.solid);
    row.limit = min(row.limit, end);
    k_lo = max(k_lo, tests.first / TK * TK);
  } else {
    tests.solid = true;  // (no key lies below tests.first = 0)
  }
  const int k_hi = min(wave_max_i(row.limit), (int)min((long)split * item.chunk + item.chunk, 0x7fffffffl));
  tests.least = wave_min_i(row.limit);
  const int tiles = k_hi > k_lo ? (k_hi - k_lo + TK - 1) / TK : 0, n_tiles = tiles > wave ? (tiles - wave + NW - 1) / NW : 0;  // this wave's: wave, wave + 4, ..

  KeyPlaces<PAGED, DH, 4> places(a, b, kvh);
  auto key_of = [&](int n) { return k_lo + (wave + n * NW) * TK; };
  float k[HALF], q[HALF], v[16][DB];
  floatx16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
  {
    const float4 *src = reinterpret_cast<const float4 *>((const float *)a.q + (size_t)place * DH + lhi * HALF);
#pragma unroll
    for (int c = 0; c < HALF / 4; ++c) {
      const float4 x = src[c];
      q[4 * c] = x.x; q[4 * c + 1] = x.y; q[4 * c + 2] = x.z; q[4 * c + 3] = x.w;
    }
  }
  size_t off[2];
  auto load_k = [&](int k0) {  // (keys past the end are the last one again, masked later)
    const int r = min(l32, k_hi - 1 - k0);
    const float4 *src = reinterpret_cast<const float4 *>(places.k + (r >= 16 ? off[1] : off[0]) + (size_t)(r & 15) * places.stride + lhi * HALF * 4);
#pragma unroll
    for (int c = 0; c < HALF / 4; ++c) {
      const float4 x = src[c];
      k[4 * c] = x.x; k[4 * c + 1] = x.y; k[4 * c + 2] = x.z; k[4 * c + 3] = x.w;
    }
  };
  auto load_v = [&](int k0) {
    const int last = k_hi - 1 - k0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = min(8 * (e / 4) + e % 4 + 4 * lhi, last);
      const unsigned char *src = places.v + (r >= 16 ? off[1] : off[0]) + (size_t)(r & 15) * places.stride + l32 * DB * 4;
      if constexpr (DB == 2) {
        const float2 x = *reinterpret_cast<const float2 *>(src);
        v[e][0] = x.x; v[e][1] = x.y;
      } else {
        const float4 x = *reinterpret_cast<const float4 *>(src);
        v[e][0] = x.x; v[e][1] = x.y; v[e][2] = x.z; v[e][3] = x.w;
      }
    }
  };
  if (n_tiles > 0) {
    places.ask(key_of(0), k_hi - 1);
    places.halves(key_of(0), off);
    load_k(key_of(0));
  }
  float m_run = -INFINITY, l_run = 0.f;
  const float sc = sh.sc;
  for (int n = 0; n < n_tiles; ++n) {
    const int k0 = key_of(n);
    load_v(k0);
    if (n + 1 < n_tiles) places.ask(key_of(n + 1), k_hi - 1);
    if (doc) {
      __builtin_amdgcn_wave_barrier();
      docs[wave][l32] = doc[min(k0 + l32, k_hi - 1)];
      __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses keep their order)
    }
    floatx16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int c = 0; c < HALF; ++c) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[c], q[c], s, 0, 0, 0);
    if (n + 1 < n_tiles) {
      places.halves(key_of(n + 1), off);
      load_k(key_of(n + 1));
    }
    const bool tested = shape_scores<DOCS_ANY>(s, sh, row, tests, k0, lhi, l32, docs[wave]);
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = xhalf_max(mx) * sc;
    // the running reference moves where the maximum exceeds it by more than 2^8: rare after the first tiles
    const bool need = mx > m_run + 8.0f;
    if (__any(need)) {
      const float corr = need ? __builtin_amdgcn_exp2f(m_run - mx) : 1.0f;
      m_run = need ? mx : m_run;
      l_run *= corr;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] *= corr;
    }
    const float neg_ref = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], sc, neg_ref));
      l_run += s[e];
    }
    if (tested) {  // values that are no finite numbers: as take_out_nonfinite
      float none = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int db = 0; db < DB; ++db) none = fmaf(v[e][db], 0.f, none);
      if (__any(none != 0.f)) {
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind) {
          const float value = __uint_as_float(kind == 0 ? 0x7fc00000u : kind == 1 ? 0x7f800000u : 0xff800000u);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            floatx16 t;
#pragma unroll
            for (int e = 0; e < 16; ++e) t[e] = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const bool is = kind == 0 ? v[e][db] != v[e][db] : v[e][db] == value;
              t = __builtin_amdgcn_mfma_f32_32x32x2f32(is ? 1.f : 0.f, s[e], t, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[db][e] += t[e] > 0.f ? value : 0.f;
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int db = 0; db < DB; ++db)
            if ((__float_as_uint(v[e][db]) & 0x7f800000u) == 0x7f800000u) v[e][db] = 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e][db], s[e], acc[db], 0, 0, 0);
  }
  l_run = xhalf_sum(l_run);
  if (PAGED && places.bad && lane == 0) *a.status = a.bad_page_code;

  // merge of the waves through LDS
  if (wave > 0) {
    float *dst = mg + (size_t)(wave - 1) * PER_WAVE + lane;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) dst[(db * 16 + e) * 64] = acc[db][e];
    dst[(DB * 16) * 64] = m_run;
    dst[(DB * 16 + 1) * 64] = l_run;
  }
  __syncthreads();
  if (wave == 0) {
    float M = m_run;
#pragma unroll
    for (int w = 0; w < NW - 1; ++w) M = fmaxf(M, mg[(size_t)w * PER_WAVE + (DB * 16) * 64 + lane]);
    const float ref = (M == -INFINITY) ? 0.f : M, c0 = __builtin_amdgcn_exp2f(m_run - ref);
    l_run *= c0;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[db][e] *= c0;
#pragma unroll
    for (int w = 0; w < NW - 1; ++w) {
      const float *src = mg + (size_t)w * PER_WAVE + lane;
      const float cw = __builtin_amdgcn_exp2f(src[(DB * 16) * 64] - ref);
      l_run = fmaf(src[(DB * 16 + 1) * 64], cw, l_run);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] = fmaf(src[(db * 16 + e) * 64], cw, acc[db][e]);
    }
    const bool whole = item.splits == 1;
    const size_t at = (size_t)split * a.cap * a.H + place;
    if (l32 < nq) {
      const float by = whole ? inverse_of(l_run) : 1.f;
      float *dst = (whole ? (float *)a.out + (size_t)place * DH : a.part_o + at * DH) + 4 * lhi * DB;  // register e of block db: column (8 (e / 4) + 4 lhi + e % 4) DB + db
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int c = 0; c < 4 * DB; c += 2) {
          const float2 x{acc[c % DB][4 * g + c / DB] * by, acc[(c + 1) % DB][4 * g + (c + 1) / DB] * by};
          if (whole) *reinterpret_cast<float2 *>(dst + 8 * g * DB + c) = x;
          else store_through(dst + 8 * g * DB + c, x);
        }
      if (!whole && lhi == 0) store_through(a.part_ml + at * 2, float2{M, l_run});
    }
  }
  if (item.splits > 1) merge_splits_last<float, DH>(a, item, red, mg);
}

template <int DH> void launch_f32(const ScoredAttn &a, hipStream_t s) {
  const int grid = (int)scored_grid(a);
  if (a.bq == 32) {
    if (a.pages.table) k_scored_f32_tile<DH, true><<<grid, 256, 0, s>>>(a);
    else k_scored_f32_tile<DH, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (a.pages.table) k_scored_f32<DH, true, 2><<<grid, 256, 0, s>>>(a);
    else k_scored_f32<DH, false, 2><<<grid, 256, 0, s>>>(a);
  }
}

// ---- work of more than 64 sequences ------------------------------------------------------------------------------
// One workgroup, a thread to a run of neighbouring sequences: the size of the pieces, then items and tiles up to every sequence by one scan.
// (With every workgroup of the attention going over all sequences instead, one token of each of 1500 requests of 512 keys, 28 heads over 4: 542 us,
// 270 with the list; of 8192 of 64 keys 8788 / 547; of 128 of 2048 88 / 88.)
constexpr int LIST_NT = 1024, LIST_NW = LIST_NT / WAVE;
__global__ __launch_bounds__(LIST_NT) void k_scored_list(ScoredAttn a) {
  __shared__ float sums[LIST_NW];
  __shared__ int ends[2][LIST_NW];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int total = scored_rows(a), per = (a.B + LIST_NT - 1) / LIST_NT, first = tid * per;
  bool down = false;
  for (int i = 0; i < per; ++i) down = down || descends(a, first + i);
  if (__syncthreads_or(down)) {  // no items
    for (int i = tid; i <= 2 * a.B; i += LIST_NT) a.list[i] = 0;
    if (tid == 0) *a.status = a.bad_offsets_code;
    return;
  }
  const int chunk = scored_chunk(a, [&](auto f) {
    float x = 0.f;
    for (int i = 0; i < per; ++i) x += f(scored_seq(a, first + i, total));  // (a sequence that is not there has no tiles)
    x = wave_fold(x, Sum{});
    if (lane == 0) sums[wave] = x;
    __syncthreads();
    x = wave_fold(lane < LIST_NW ? sums[lane] : 0.f, Sum{});
    __syncthreads();
    return x;
  });
  int n[2] = {0, 0};
  for (int i = 0; i < per; ++i) {
    const ScoredSeq q = scored_seq(a, first + i, total);
    n[0] += q.tiles * split_count(q.keys, split_size(a, q.keys, chunk));
    n[1] += q.tiles;
  }
  int upto[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    upto[k] = wave_scan(n[k]);
    if (lane == WAVE - 1) ends[k][wave] = upto[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int waves = wave_scan(lane < LIST_NW ? ends[k][lane] : 0);
    upto[k] += (wave ? __builtin_amdgcn_readlane(waves, wave - 1) : 0) - n[k];
  }
  if (tid == 0) a.list[0] = chunk;
  int32_t *items_to = a.list + LIST_HEAD, *tiles_to = items_to + a.B;
  for (int i = 0; i < per && first + i < a.B; ++i) {
    const ScoredSeq q = scored_seq(a, first + i, total);
    upto[0] += q.tiles * split_count(q.keys, split_size(a, q.keys, chunk));
    upto[1] += q.tiles;
    items_to[first + i] = upto[0];
    tiles_to[first + i] = upto[1];
  }
}

// ---- merge of the splits of many rows: a wave to a (row, head), its lanes the splits' weights, then the columns ------------
// Bound by the latency of its dependent reads.
template <int DH>
__global__ __launch_bounds__(256) void k_scored_merge(ScoredAttn a) {
  constexpr int V = DH / WAVE;
  if (no_order(a)) return;
  const int n = scored_rows(a), lane = threadIdx.x % WAVE;
  const uint32_t items = (uint32_t)n * (uint32_t)a.H, first = a.offsets ? (uint32_t)max(a.offsets[0], 0) * (uint32_t)a.H : 0u;  // (rows ahead are no sequence's)
  const size_t step = (size_t)a.cap * a.H;
  for (uint32_t it = first + blockIdx.x * 4 + threadIdx.x / WAVE; it < items; it += gridDim.x * 4) {
    const int splits = min(a.n_split[it / (uint32_t)a.H], a.splits);
    if (splits <= 1) continue;  // (the row is finished)
    float m[2], l[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int s = lane + u * WAVE;
      const float2 ml = s < splits ? *reinterpret_cast<const float2 *>(a.part_ml + ((size_t)s * step + it) * 2) : float2{-INFINITY, 0.f};
      m[u] = ml.x; l[u] = ml.y;
    }
    const float M = wave_max(fmaxf(m[0], m[1])), ref = M == -INFINITY ? 0.f : M;
    float w[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) w[u] = __builtin_amdgcn_exp2f(m[u] - ref);
    const float inv = inverse_of(wave_sum(l[0] * w[0] + l[1] * w[1]));
    float o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = 0.f;
    const float *po = a.part_o + (size_t)it * DH + lane * V;
    auto weight = [&](int s) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s < WAVE ? w[0] : w[1]), s % WAVE)); };
    for (int s0 = 0; s0 < splits; s0 += 8) {  // (eight loads in flight; past the end the last split again, with no weight)
      float x[8][V];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][e] = po[(size_t)min(s0 + i, splits - 1) * step * DH + e];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (s0 + i >= splits) break;  // uniform
        const float ws = weight(s0 + i);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(x[i][e], ws, o[e]);
      }
    }
    bf16_t *out = (bf16_t *)a.out + (size_t)it * DH + lane * V;
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = f2bf(o[e] * inv);
  }
}

void launch_merge(const ScoredAttn &a, hipStream_t s) {
  const long blocks = ((long)a.cap * a.H + 3) / 4;
  const int grid = (int)(blocks > 8192 ? 8192 : blocks);
  if (a.dh == 64) k_scored_merge<64><<<grid, 256, 0, s>>>(a);
  else k_scored_merge<128><<<grid, 256, 0, s>>>(a);
}

}  // namespace

// Rows of a workgroup and key splits, of what the host knows: the list's capacity stands for its count, the room of the caches for the lengths.
// The prices are fits to launches of 1 to 16 sequences of 512 to 8192 keys and 1 to 100 rows (32 heads of 128, 28 over 4, 8 over 2 of 64), ns of a key
// of a sequence: in a workgroup that has its CU alone, what each adds where there are more than CUs, and the way of all keys from memory.
// Of nine choices each (both forms, 1 split or about 128, 256, 384 and 512 workgroups) the one taken is 4 % slower than the best in the geometric
// mean of 108 shapes.  (Beyond two workgroups a CU pieces pay only where without them a few CUs had two: one token of 66 requests of 4096 keys, 4 heads,
// 150 -> 111 us; of 9 of 8192, 32 heads, 263 -> 199; but of 100 of 2048, 4 heads, 73 -> 88, which the 1.15 keeps whole.)  A few, 32 / 128 rows without splits / as chosen, us: one token of one sequence of 8192 keys, 32 heads, 85 / 126 / 31; in each of
// 16, 28 heads over 4, 91 / 127 / 51; 100 rows of each of 16 of 2048 159 / 68 / 68; 8 heads over 2 of 64, 100 rows of 2048 keys 19.4 / 33 / 17.
// fp32, by 90 shapes of the same kind: two rows a workgroup until there are many, then 32; the one taken is 4 % slower than the best of eight.
void scored_plan(DType t, ScoredAttn *a) {
  const long g = a->H / a->Hkv, rows = a->offsets ? ((long)a->cap + a->B - 1) / a->B : a->L, packed = rows * g;
  const bool d128 = a->dh == 128;
  const size_t per_split = (size_t)a->cap * a->H * a->dh;
  long most = (long)(a->part_elems / (per_split ? per_split : 1));
  most = std::min({most, (long)MAX_SPLITS, (a->L + SPLIT_KEYS - 1l) / SPLIT_KEYS});
  struct Form { int bq; double alone, each, memory; };  // memory: bytes a ns of the whole chip
  const Form forms_f32[2] = {{2, d128 ? 18.7 : 9.3, d128 ? 0.07 : 0.037, 6000}, {32, d128 ? 40. : 21., d128 ? 0.155 : 0.083, 5000}};
  const Form forms_bf16[2] = {{32, d128 ? 9.4 : 6.2, d128 ? 0.05 : 0.021, 5000}, {128, d128 ? 14.4 : 11.2, d128 ? 0.06 : 0.032, 5600}};
  const Form *forms = t == F32 ? forms_f32 : forms_bf16;
  double best = 0;
  for (int i = 0; i < 2; ++i) {
    const Form &f = forms[i];
    const double n = (double)a->B * a->Hkv * ((packed + f.bq - 1) / f.bq);
    const double memory = (double)a->B * a->Hkv * a->dh * (t == F32 ? 8 : 4) / f.memory;
    const bool fused = packed <= FUSED_ROWS || t == F32;
    for (int s = 1; s == 1 || s <= most; s += s < 8 ? 1 : s / 4) {
      const double m = n * s;
      if (s > 1 && (m > 1024 || (!fused && a->cap > a->split_rows))) break;
      const double rounds = f.each * (m > 256 ? 256 * ceil(m / 256) : m);  // (a CU with two workgroups where others have one ends last)
      const double work = (rounds > f.alone ? rounds : f.alone) / s, way = memory * (m < 160 ? 1.6 : m < 256 ? 256 / m : m > 512 && s > 1 ? 1.15 : 1);  // (few workgroups draw less; a second round costs a start)
      const double ends = a->kv_len ? 1 + 0.25 / s : 1;  // (of ragged sequences the last pieces are half empty)
      const double merge = s == 1 ? 0 : !fused ? 6000 + 60.0 * s + (double)per_split * (s * 8 / 3000. + 0.4 / a->dh)
                                  : packed <= FUSED_ROWS || f.bq <= FUSED_ROWS ? 1500 + 100.0 * s * std::min(packed, (long)FUSED_ROWS) / FUSED_ROWS
                                  : 1500 + (std::min(packed, (long)f.bq) + FUSED_ROWS - 1) / FUSED_ROWS * (2000 + 100.0 * s) + (double)per_split * (s * 8 / 3000.);
      const double ns = a->L * (work > way ? work : way) * ends + merge;
      if (i == 0 && s == 1 ? true : ns < best) {
        best = ns;
        a->bq = f.bq; a->fused = fused;
        a->splits = s > 1 ? (int)most : 1;
        a->target = (int)m;
      }
    }
  }
  if (a->fused && scored_tiles(*a) * a->Hkv > ARRIVE_WORDS) a->splits = 1;
  if (a->fused || a->splits == 1) a->n_split = nullptr;
  // Keys and values that at most two tiles of a sequence read displace others in the L2 for nothing: 16 x 1280 keys, 77 rows each, 79.9 -> 71.1 us; 32 rows
  // 59.3 -> 51.2; one token of 32 requests of 11000 to 32768 keys, 28 heads over 4, 267 -> 243.  With more tiles the later ones find them there:
  // 4 chunks of 2048 rows 515 -> 555.  Small caches make no difference (one token of 8 x 8192 keys of 2 heads of 64 18.9 -> 18.4).
  a->once = a->bq == 128 && packed * 2 <= 3 * 128 && (size_t)a->B * a->L * a->Hkv * a->dh * 4 >= (size_t)32 << 20;
}

void launch_attention_scored(DType t, const ScoredAttn &a, hipStream_t s) {
  if (a.cap <= 0) return;
  if (a.B > WAVE) k_scored_list<<<1, LIST_NT, 0, s>>>(a);
  if (t == F32) {
    if (a.dh == 64) launch_f32<64>(a, s);
    else launch_f32<128>(a, s);
  } else if (a.pages.table) {
    if (a.bq == 32) launch_scored_pages_few(a, s);
    else if (a.once) launch_scored_pages_once(a, s);
    else launch_scored_pages_many(a, s);
  } else {
    if (a.bq == 32) launch_scored_dense_few(a, s);
    else if (a.once) launch_scored_dense_once(a, s);
    else launch_scored_dense_many(a, s);
  }
  if (a.n_split) launch_merge(a, s);
}

}  // namespace dy
