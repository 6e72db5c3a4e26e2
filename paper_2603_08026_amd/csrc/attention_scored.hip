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
// registers, a step ahead, the pages' numbers another.  Every product and sum is fp32.
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

template <int DH, int R> void launch_f32(const ScoredAttn &a, hipStream_t s) {
  if (a.pages.table) k_scored_f32<DH, true, R><<<(int)scored_grid(a), 256, 0, s>>>(a);
  else k_scored_f32<DH, false, R><<<(int)scored_grid(a), 256, 0, s>>>(a);
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
  const int n = scored_rows(a), lane = threadIdx.x % WAVE;
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
void scored_plan(DType t, ScoredAttn *a) {
  const long g = a->H / a->Hkv, rows = a->offsets ? ((long)a->cap + a->B - 1) / a->B : a->L, packed = rows * g;
  const bool d128 = a->dh == 128;
  const size_t per_split = (size_t)a->cap * a->H * a->dh;
  long most = (long)(a->part_elems / (per_split ? per_split : 1));
  most = std::min({most, (long)MAX_SPLITS, (a->L + SPLIT_KEYS - 1l) / SPLIT_KEYS});
  struct Form { int bq; double alone, each, memory; };  // memory: bytes a ns of the whole chip
  const Form forms_f32[1] = {{2, d128 ? 18.7 : 9.3, d128 ? 0.07 : 0.037, 6000}};
  const Form forms_bf16[2] = {{32, d128 ? 9.4 : 6.2, d128 ? 0.05 : 0.021, 5000}, {128, d128 ? 14.4 : 11.2, d128 ? 0.06 : 0.032, 5600}};
  const Form *forms = t == F32 ? forms_f32 : forms_bf16;
  double best = 0;
  for (int i = 0; i < (t == F32 ? 1 : 2); ++i) {
    const Form &f = forms[i];
    const double n = (double)a->B * a->Hkv * ((packed + f.bq - 1) / f.bq);
    const double memory = (double)a->B * a->Hkv * a->dh * (t == F32 ? 8 : 4) / f.memory;
    const bool fused = packed <= FUSED_ROWS || f.bq <= FUSED_ROWS;
    for (int s = 1; s == 1 || s <= most; s += s < 8 ? 1 : s / 4) {
      const double m = n * s;
      if (s > 1 && (m > 1024 || (!fused && a->cap > a->split_rows))) break;
      const double rounds = f.each * (m > 256 ? 256 * ceil(m / 256) : m);  // (a CU with two workgroups where others have one ends last)
      const double work = (rounds > f.alone ? rounds : f.alone) / s, way = memory * (m < 160 ? 1.6 : m < 256 ? 256 / m : m > 512 && s > 1 ? 1.15 : 1);  // (few workgroups draw less; a second round costs a start)
      const double ends = a->kv_len ? 1 + 0.25 / s : 1;  // (of ragged sequences the last pieces are half empty)
      const double merge = s == 1 ? 0 : fused ? 1500 + 100.0 * s * (packed < 8 ? packed : 8) / 8
                                              : 6000 + 60.0 * s + (double)per_split * (s * 8 / 3000. + 0.4 / a->dh);
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
    if (a.dh == 64) launch_f32<64, 2>(a, s);
    else launch_f32<128, 2>(a, s);
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
