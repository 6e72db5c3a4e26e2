// Attention with masked and reshaped scores: fp32, the merge of key splits, and which kernel takes a call.
#include "attention_scored.h"
#include <float.h>

namespace dy {

namespace {

// ---- fp32: R packed rows a workgroup ------------------------------------------------------------------------------
// dh / 16 lanes take a key, a lane 16 of its elements, and 64 / (dh / 16) keys go through a wave at a time, each group of lanes with a running
// maximum, sum and result of its own; four waves take such steps in turn, and groups and waves are merged at the end.  Every product is fp32.
template <int DH, bool PAGED, int R>
__global__ __launch_bounds__(256, 2) void k_scored_f32(ScoredAttn a) {
  constexpr int CPK = DH / 16, KS = WAVE / CPK, NW = 4;  // lanes of a key, keys of a wave's step, waves
  __shared__ float part[NW][R][DH], part_ml[NW][R][2];
  __shared__ int red[2 * NW];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int c = lane % CPK, group = lane / CPK;
  const ScoredItem item = scored_item(a, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such item
  const int nq = item.n, grp = a.H / a.Hkv;
  auto row_of = [&](int r) { return item.row + (item.packed + r) / grp; };
  auto head_of = [&](int r) { return kvh * grp + (item.packed + r) % grp; };
  auto place = [&](int r) { return (uint32_t)row_of(r) * (uint32_t)a.H + (uint32_t)head_of(r); };
  RowMask row[R];
  int k_lo = split * item.chunk, k_hi = 0, lo = 0x7fffffff, hi = -1;
  const int32_t *docs = a.doc ? a.doc + (size_t)b * a.L : nullptr;
#pragma unroll
  for (int r = 0; r < R; ++r) {  // (rows past the end: the last one again, their results are never stored)
    const int rr = min(r, nq - 1), i = position_of(a, PAGED, b, row_of(rr));
    row[r].limit = limit_of(a, b, item.keys, i);
    row[r].pos = (float)i;
    row[r].slope = a.slopes ? a.slopes[head_of(rr)] * LOG2E : 0.f;
    if (docs) {
      row[r].doc = i >= 0 && i < a.L ? docs[i] : -1;
      if (row[r].doc < 0) row[r].limit = 0;
      lo = min(lo, row[r].doc < 0 ? 0x7fffffff : row[r].doc);
      hi = max(hi, row[r].doc);
    }
    k_hi = max(k_hi, row[r].limit);
  }
  k_hi = min(k_hi, (int)min((long)k_lo + item.chunk, 0x7fffffffl));
  if (docs) {
    int first, end;
    doc_range(docs, item.keys, lo, hi, red, &first, &end);
    k_hi = min(k_hi, end);
    k_lo = max(k_lo, first);
  }
  const Shape sh(a);
  float q[R][16], acc[R][16], m_run[R], l_run[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float4 *src = reinterpret_cast<const float4 *>((const float *)a.q + (size_t)place(min(r, nq - 1)) * DH + c * 16);
    const float by = sh.capped ? 1.f : sh.sc;  // scores are kept in the log2 domain
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = src[i];
      q[r][4 * i] = x.x * by; q[r][4 * i + 1] = x.y * by; q[r][4 * i + 2] = x.z * by; q[r][4 * i + 3] = x.w * by;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[r][e] = 0.f;
    m_run[r] = -FLT_MAX;  // (finite, so that a score of -inf has the probability 0)
    l_run[r] = 0.f;
  }
  const size_t dense = ((size_t)b * a.L * a.Hkv + kvh) * DH + c * 16, head = ((size_t)kvh << a.pages.shift) * DH + c * 16;
  const int32_t *table = PAGED ? a.pages.table + (size_t)b * a.pages.max_pages : nullptr;
  bool bad = false;
  struct Step { float k[16], v[16]; int doc; };
  auto key_of = [&](int n) { return k_lo + (n * NW + wave) * KS + group; };
  auto load = [&](int n, Step &s) {  // (keys past the end: the last one again, masked later)
    const int key = min(key_of(n), k_hi - 1);
    size_t at;
    if constexpr (PAGED) {
      int page = table[key >> a.pages.shift];
      if ((uint32_t)page >= (uint32_t)a.pages.n_pages) { page = 0; bad = true; }
      at = (((size_t)(uint32_t)page * a.Hkv) << a.pages.shift) * DH + head + (size_t)(key & ((1 << a.pages.shift) - 1)) * DH;
    } else {
      at = dense + (size_t)key * a.Hkv * DH;
    }
    const float4 *ks = reinterpret_cast<const float4 *>((const float *)(PAGED ? a.pages.k : a.k) + at);
    const float4 *vs = reinterpret_cast<const float4 *>((const float *)(PAGED ? a.pages.v : a.v) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = ks[i], y = vs[i];
      s.k[4 * i] = x.x; s.k[4 * i + 1] = x.y; s.k[4 * i + 2] = x.z; s.k[4 * i + 3] = x.w;
      s.v[4 * i] = y.x; s.v[4 * i + 1] = y.y; s.v[4 * i + 2] = y.z; s.v[4 * i + 3] = y.w;
    }
    s.doc = docs ? docs[key] : 0;
  };
  const int n_steps = k_hi > k_lo ? (k_hi - k_lo + NW * KS - 1) / (NW * KS) : 0;
  Step next;
  if (n_steps > 0) load(0, next);
  for (int n = 0; n < n_steps; ++n) {
    Step now = next;
    if (n + 1 < n_steps) load(n + 1, next);
    const int key = key_of(n);
    float score[R];
    bool need = false, all = true;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float d0 = 0.f, d1 = 0.f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        d0 = fmaf(q[r][e], now.k[e], d0);
        d1 = fmaf(q[r][e + 1], now.k[e + 1], d1);
      }
      float x = lanes_sum<CPK>(d0 + d1);
      if (sh.capped) x = sh.cap_out * tanhf(x * (sh.sc / sh.cap_out));
      if (sh.sloped) x = fmaf(-row[r].slope, fabsf(row[r].pos - (float)key), x);
      const bool counts = key < k_hi && key < row[r].limit && (!docs || now.doc == row[r].doc);
      all = all && counts;
      score[r] = counts ? x : -INFINITY;
      need = need || score[r] > m_run[r] + 8.0f;
    }
    if (__any(need)) {  // the running reference moves where a score exceeds it by more than 2^8: rare after the first steps
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float top = fmaxf(m_run[r], score[r]);
        const float corr = __builtin_amdgcn_exp2f(m_run[r] - top);
        m_run[r] = top;
        l_run[r] *= corr;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][e] *= corr;
      }
    }
    if (__all(all)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float p = __builtin_amdgcn_exp2f(score[r] - m_run[r]);
        l_run[r] += p;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][e] = fmaf(p, now.v[e], acc[r][e]);
      }
    } else {  // (a value that does not count may be no number)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool counts = score[r] != -INFINITY;
        const float p = counts ? __builtin_amdgcn_exp2f(score[r] - m_run[r]) : 0.f;
        l_run[r] += p;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][e] = fmaf(p, counts ? now.v[e] : 0.f, acc[r][e]);
      }
    }
  }
  if (PAGED && bad) *a.status = a.bad_page_code;
  // merge of a wave's groups: each exchange halves the elements that a lane answers for
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float top = m_run[r];
#pragma unroll
    for (int off = CPK; off < WAVE; off *= 2) top = fmaxf(top, __shfl_xor(top, off, WAVE));
    const float by = __builtin_amdgcn_exp2f(m_run[r] - top);
    float l = l_run[r] * by;
#pragma unroll
    for (int off = CPK; off < WAVE; off *= 2) l += __shfl_xor(l, off, WAVE);
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[r][e] *= by;
    int col = c * 16;
#pragma unroll
    for (int off = WAVE / 2, half = 8; off >= CPK; off /= 2, half /= 2) {
      const bool up = lane & off;
#pragma unroll
      for (int e = 0; e < half; ++e) {
        const float keep = up ? acc[r][e + half] : acc[r][e], send = up ? acc[r][e] : acc[r][e + half];
        acc[r][e] = keep + __shfl_xor(send, off, WAVE);
      }
      col += up ? half : 0;
    }
#pragma unroll
    for (int e = 0; e < 16 / KS; ++e) part[wave][r][col + e] = acc[r][e];
    if (lane == 0) {
      part_ml[wave][r][0] = top;
      part_ml[wave][r][1] = l;
    }
  }
  __syncthreads();
  // merge of the waves
  const bool whole = item.splits == 1;
  if (a.splits > 1 && kvh == 0 && split == 0 && tid < nq) a.n_split[row_of(tid)] = item.splits;
  for (int i = tid; i < nq * DH; i += 256) {
    const int r = i / DH, col = i % DH;
    float top = part_ml[0][r][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, part_ml[w][r][0]);
    float o = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float by = __builtin_amdgcn_exp2f(part_ml[w][r][0] - top);
      o = fmaf(part[w][r][col], by, o);
      l = fmaf(part_ml[w][r][1], by, l);
    }
    const size_t at = place(r) + (whole ? 0 : (size_t)split * a.cap * a.H);
    if (whole) {
      ((float *)a.out)[at * DH + col] = l == 0.f ? 0.f : o / l;
    } else {  // (a split without keys counts for nothing)
      a.part_o[at * DH + col] = o;
      if (col == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{l == 0.f ? -INFINITY : top, l};
    }
  }
}

template <int DH, int R> void launch_f32(const ScoredAttn &a, hipStream_t s) {
  if (a.pages.table) k_scored_f32<DH, true, R><<<(int)scored_grid(a), 256, 0, s>>>(a);
  else k_scored_f32<DH, false, R><<<(int)scored_grid(a), 256, 0, s>>>(a);
}

// ---- merge of the splits: a wave to a (row, head), its lanes the splits' weights, then the columns --------------------
constexpr int MAX_SPLITS = 128;
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_scored_merge(ScoredAttn a) {
  constexpr int V = DH / WAVE;
  const int n = a.offsets ? min(a.offsets[a.B], a.cap) : a.cap, lane = threadIdx.x % WAVE;
  const uint32_t items = (uint32_t)n * (uint32_t)a.H;
  const size_t step = (size_t)a.cap * a.H;
  for (uint32_t it = blockIdx.x * 4 + threadIdx.x / WAVE; it < items; it += gridDim.x * 4) {
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
    const float total = wave_sum(l[0] * w[0] + l[1] * w[1]);
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
        const float ws = s0 + i < splits ? weight(s0 + i) : 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = s0 + i < splits ? fmaf(x[i][e], ws, o[e]) : o[e];
      }
    }
    const float inv = inverse_of(total);
    T *out = (T *)a.out + (size_t)it * DH + lane * V;
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = from_f<T>(o[e] * inv);
  }
}

template <typename T> void launch_merge(const ScoredAttn &a, hipStream_t s) {
  const long blocks = ((long)a.cap * a.H + 3) / 4;
  const int grid = (int)(blocks > 8192 ? 8192 : blocks);
  if (a.dh == 64) k_scored_merge<T, 64><<<grid, 256, 0, s>>>(a);
  else k_scored_merge<T, 128><<<grid, 256, 0, s>>>(a);
}

}  // namespace

// Rows of a workgroup and key splits, of what the host knows: the list's capacity stands for its count.
void scored_plan(DType t, ScoredAttn *a) {
  const long g = a->H / a->Hkv, rows = a->offsets ? ((long)a->cap + a->B - 1) / a->B : a->L, packed = rows * g;
  auto items = [&](int bq) { return (long)a->B * a->Hkv * ((packed + bq - 1) / bq); };
  const int few = t == F32 ? 1 : 32, many = t == F32 ? 4 : 128;
  a->bq = t == F32 ? (items(4) >= 1024 ? many : few) : packed > 48 && items(128) >= 128 ? many : few;
  a->target = 512;
  const size_t per_split = (size_t)a->cap * a->H * a->dh;
  const long room = (long)(a->part_elems / (per_split ? per_split : 1)), by_keys = (a->L + SPLIT_KEYS - 1) / SPLIT_KEYS;
  long splits = room < MAX_SPLITS ? room : MAX_SPLITS;
  if (splits > by_keys) splits = by_keys;
  a->splits = items(a->bq) * 4 > a->target * 3 || splits < 2 ? 1 : (int)splits;
}

void launch_attention_scored(DType t, const ScoredAttn &a, hipStream_t s) {
  if (a.cap <= 0) return;
  if (t == F32) {
    if (a.dh == 64 && a.bq == 1) launch_f32<64, 1>(a, s);
    else if (a.dh == 64) launch_f32<64, 4>(a, s);
    else if (a.bq == 1) launch_f32<128, 1>(a, s);
    else launch_f32<128, 4>(a, s);
    if (a.splits > 1) launch_merge<float>(a, s);
    return;
  }
  if (a.pages.table) {
    if (a.bq == 32) launch_scored_pages_few(a, s);
    else launch_scored_pages_many(a, s);
  } else {
    if (a.bq == 32) launch_scored_dense_few(a, s);
    else launch_scored_dense_many(a, s);
  }
  if (a.splits > 1) launch_merge<bf16_t>(a, s);
}

}  // namespace dy
