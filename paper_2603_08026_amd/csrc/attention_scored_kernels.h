// The two bf16 kernels of attention with masked and reshaped scores (attention_scored.h), for 32 and for 128 packed query rows a workgroup.  Products
// are transposed as in attention_bf16.hip: S^T = K Q^T, O^T = V^T P^T, a lane has one query, and P^T goes from one product to the next in
// registers.  Probabilities are rounded to the bf16 of the matrix instruction and sums are taken over the rounded ones; everything else is fp32.
#pragma once
#include "attention_scored.h"

namespace dy {

namespace {

// ---- 32 packed rows a workgroup: few rows ----------------------------------------------------------------------
// Bound by the keys' and values' way from memory.  The four waves share nothing: each streams key tiles of its own (tile wave, wave + 4, ..) through
// its own ring in LDS, with no barrier in the loop; their results are merged once at the end.  8 rows of each of 4 sequences of 512 keys, 32 heads of 128, 14.0 us
// where the tile of 128 takes 16.6; from long sequences that tile's copies past the L2, two workgroups a CU, draw more.
template <int DH, int MODE> struct FewTile : KeyTile<DH> {
  using K = KeyTile<DH>;
  static constexpr int NW = 4, NS = DH == 128 ? 2 : 4, BQ = 32;
  static constexpr int STAGE = 2 * K::REGION + (MODE & DOCS ? 256 : 0), PER_TILE = 2 * K::COPIES + (MODE & DOCS ? 1 : 0);
  static constexpr int PER_WAVE = (K::DB * 16 + 2) * 64;  // floats of a wave's result
  static constexpr int RING = NS * STAGE, LDS = NW * RING;
  static_assert((NS - 1) * PER_TILE < 64 && (NW - 1) * PER_WAVE * 4 <= LDS && LDS <= 160 * 1024, "vmcnt immediate, merge scratch");
};

template <int DH, bool PAGED, int MODE>
__global__ __launch_bounds__(256, 1) void k_scored_few(ScoredAttn a) {
  using T = FewTile<DH, MODE>;
  constexpr int TK = T::TK, ROWB = T::ROWB, DB = T::DB, KK = T::KK, CH = T::CH, RPC = T::RPC, NW = T::NW, NS = T::NS, COPIES = T::COPIES;
  __shared__ __align__(1024) unsigned char smem[T::LDS];
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
  const Shape sh(a);
  RowMask row;
  TileTests tests;
  int k_lo = split * item.chunk, k_hi;
  {
    const int i = position_of(a, PAGED, b, jq);
    row.limit = limit_of(a, b, item.keys, i);
    row.pos = i;
    if ((MODE & BIASED) && a.slopes) row.slope = sh.slope(a.slopes[hq]);
    if constexpr (MODE & DOCS) {
      row.doc = i >= 0 && i < a.L ? a.doc[(size_t)b * a.L + i] : -1;
      if (row.doc < 0) row.limit = 0;
      const int some = row.doc < 0 ? 0x7fffffff : row.doc, lo = wave_min_i(some), hi = wave_max_i(row.doc);
      tests.one = __all(row.doc == hi);
      int end;
      doc_range(a.doc + (size_t)b * a.L, item.keys, lo, hi, red, &tests.first, &end, &tests.solid);
      row.limit = min(row.limit, end);  // (the sweep ends there, in the middle of a tile)
    }
    k_hi = min(wave_max_i(row.limit), (int)min((long)k_lo + item.chunk, 0x7fffffffl));
    if (MODE & DOCS) k_lo = max(k_lo, tests.first / TK * TK);
    tests.least = wave_min_i(row.limit);
  }
  const int tiles = k_hi > k_lo ? (k_hi - k_lo + TK - 1) / TK : 0, n_tiles = tiles > wave ? (tiles - wave + NW - 1) / NW : 0;  // this wave's: wave, wave + 4, ..

  unsigned char *own = smem + wave * T::RING;
  const uint32_t lds0 = lds_offset_of(own);
  KeyPlaces<PAGED, DH> places(a, b, kvh);
  auto key_of = [&](int n) { return k_lo + (wave + n * NW) * TK; };
  uint32_t off_k[COPIES], off_v[COPIES];  // of a full tile
#pragma unroll
  for (int i = 0; i < COPIES; ++i) {
    const int r = i * RPC + lane / CH;
    off_k[i] = (uint32_t)(r & 15) * places.stride + T::k_chunk(r, lane % CH) * 16u;
    off_v[i] = (uint32_t)(r & 15) * places.stride + T::v_chunk(r, lane % CH) * 16u;
  }
  // keys past the end are the last one again, masked later
  auto issue = [&](int n) {
    const uint32_t base = lds0 + (uint32_t)(n % NS) * T::STAGE;
    const int k0 = key_of(n), last = k_hi - 1 - k0;
    size_t off[2];
    places.halves(k0, off);
    if (last >= TK - 1) {  // uniform
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        const size_t o = off[i * RPC / 16];
        dma16_s(places.k + o, off_k[i], __builtin_amdgcn_readfirstlane(base + i * 1024u));
        dma16_s(places.v + o, off_v[i], __builtin_amdgcn_readfirstlane(base + T::REGION + i * 1024u));
      }
    } else {
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        const int to = i * RPC + lane / CH, r = min(to, last);
        const size_t o = (r >= 16 ? off[1] : off[0]) + (size_t)(r & 15) * places.stride;
        dma16(places.k + o + T::k_chunk(to, lane % CH) * 16, base + i * 1024u);
        dma16(places.v + o + T::v_chunk(to, lane % CH) * 16, base + T::REGION + i * 1024u);
      }
    }
    if constexpr (MODE & DOCS) dma4(a.doc + (size_t)b * a.L + k0 + min(l32, last), base + 2 * T::REGION);
  };
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < n_tiles) {
      places.ask(key_of(s), k_hi - 1);
      issue(s);
    }
  if (NS < n_tiles) places.ask(key_of(NS), k_hi - 1);

  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>((const bf16_t *)a.q + (size_t)place * DH + lhi * 8 + kk * 16);
  floatx16 acc_o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[db][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float sc = sh.sc;
  const int vrow = 4 * lhi + (lane % 16) / 4, hb = (lane / 16) & 1;

  for (int n = 0; n < n_tiles; ++n) {
    // tile n has landed, of those up to n + NS - 1 that exist
    if (n + NS - 1 < n_tiles) wait_vmcnt<(NS - 1) * T::PER_TILE>();
    else if (NS > 3 && n + 2 < n_tiles) wait_vmcnt<2 * T::PER_TILE>();
    else if (NS > 2 && n + 1 < n_tiles) wait_vmcnt<T::PER_TILE>();
    else wait_vmcnt<0>();
    const unsigned char *st = own + (n % NS) * T::STAGE;
    floatx16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(st + l32 * ROWB + T::k_chunk(l32, 2 * kk + lhi) * 16);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], s, 0, 0, 0);
    }
    bf16x8 vf[2][DB], pf[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const unsigned char *at = st + T::REGION + (vrow + 16 * ks) * ROWB + T::v_pair(vrow, db * 2 + hb) * 32 + 8 * (lane % 4);
        const shortx4 g0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at));
        const shortx4 g1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at + 8 * ROWB));
        vf[ks][db] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(g0, g1, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    const bool tested = shape_scores<MODE>(s, sh, row, tests, key_of(n), lhi, l32, reinterpret_cast<const int32_t *>(st + 2 * T::REGION));
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
        for (int e = 0; e < 16; ++e) acc_o[db][e] *= corr;
    }
    const float neg_ref = m_run == -INFINITY ? 0.f : -m_run;
    const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3f803f80u);
    uint32_t pw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      pw[i] = pack_bf16(__builtin_amdgcn_exp2f(fmaf(s[2 * i], sc, neg_ref)), __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], sc, neg_ref)));
      l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pw[i]), ones, l_run, false);
    }
    pf[0] = __builtin_bit_cast(bf16x8, uint4{pw[0], pw[1], pw[2], pw[3]});
    pf[1] = __builtin_bit_cast(bf16x8, uint4{pw[4], pw[5], pw[6], pw[7]});
    if (n + NS < n_tiles) {
      wait_lgkmcnt0();  // tile n has been read: another may come in its place
      issue(n + NS);
      if (n + NS + 1 < n_tiles) places.ask(key_of(n + NS + 1), k_hi - 1);
    }
    if (tested) take_out_nonfinite<DB>(vf, pf, acc_o);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][db], pf[ks], acc_o[db], 0, 0, 0);
  }
  l_run = xhalf_sum(l_run);
  if (PAGED && places.bad && lane == 0) *a.status = a.bad_page_code;

  // merge of the waves through LDS
  float *mg = reinterpret_cast<float *>(smem);
  __syncthreads();
  if (wave > 0) {
    float *dst = mg + (size_t)(wave - 1) * T::PER_WAVE + lane;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) dst[(db * 16 + e) * 64] = acc_o[db][e];
    dst[(DB * 16) * 64] = m_run;
    dst[(DB * 16 + 1) * 64] = l_run;
  }
  __syncthreads();
  if (wave > 0 && (item.splits == 1 || !a.fused)) return;
  if (wave == 0) {
    float M = m_run;
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, mg[(size_t)(w - 1) * T::PER_WAVE + (DB * 16) * 64 + lane]);
    const float ref = (M == -INFINITY) ? 0.f : M;
    const float c0 = __builtin_amdgcn_exp2f(m_run - ref);
    l_run *= c0;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc_o[db][e] *= c0;
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      const float *src = mg + (size_t)(w - 1) * T::PER_WAVE + lane;
      const float cw = __builtin_amdgcn_exp2f(src[(DB * 16) * 64] - ref);
      l_run = fmaf(src[(DB * 16 + 1) * 64], cw, l_run);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc_o[db][e] = fmaf(src[(db * 16 + e) * 64], cw, acc_o[db][e]);
    }
    if (a.n_split && kvh == 0 && split == 0 && lhi == 0 && l32 < nq) a.n_split[jq] = item.splits;
    if (item.splits > 1) {
      if (l32 < nq) store_scored_partial<DH>(a, acc_o, item, place, jq, lhi, M, l_run);
    } else if (l32 < nq) {
      const float inv = inverse_of(l_run);
      bf16_t *out = (bf16_t *)a.out + (size_t)place * DH + 4 * lhi;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<uint2 *>(out + db * 32 + 8 * g) =
              uint2{pack_bf16(acc_o[db][4 * g] * inv, acc_o[db][4 * g + 1] * inv), pack_bf16(acc_o[db][4 * g + 2] * inv, acc_o[db][4 * g + 3] * inv)};
    }
  }
  if (item.splits > 1 && a.fused) merge_splits_last<bf16_t, DH>(a, item, red, mg);
}

// ---- 128 packed rows a workgroup: many rows ----------------------------------------------------------------------
// Four waves of 32 rows over shared tiles of 32 keys, four stages in LDS, two workgroups a CU; the loop is that of k_attn_bf16_dma: while the
// vector ALU takes the exponentials of tile t, the matrix pipe works through P V of tile t - 1 and the scores of tile t + 1, and the copies of tile
// t + 3 go out one behind each few products.  Tiles that need no test run in a loop unrolled over the stages; a tile that may need one, and the last
// ones, in a body with the tests.  Bound by the exponentials beside the matrix pipe: 4096 rows of 4096 keys without masks 1090 to 1140 TFLOP/s, what the
// library's product of 8192 x 8192 matrices reaches; 4 chunks of 2048 rows in causal order over up to 8192 keys 514 to 530 us, 940 to 967 TFLOP/s of what counts (the
// tiles on the diagonal are whole).  Few rows: by the way from memory, one token of 32 requests of 11000 to 32768 keys, 28 heads over 4, 236 us, 6.3 TB/s.
// (Documents with heads of 128 spill 9 vector registers, all outside the loops.)
template <int DH, int MODE> struct ManyTile : KeyTile<DH> {
  using K = KeyTile<DH>;
  static constexpr int NW = 4, NS = 4, BQ = 128;
  static constexpr int STAGE = 2 * K::REGION + (MODE & DOCS ? NW * 256 : 0);
  static constexpr int CPW = K::COPIES / NW, LPW = 2 * CPW + (MODE & DOCS ? 1 : 0);  // copies a wave and tile
  static constexpr int SLOTS = K::DB + K::KK, LDS = NS * STAGE;
  static_assert(CPW >= 1 && (NS - 2) * LPW < 64 && LDS <= 80 * 1024 && BQ * K::ROWB <= LDS, "two workgroups a CU; rows leave by way of the same memory");
};

// ONCE: keys and values are copied past the L2.
template <int DH, bool PAGED, int MODE, bool ONCE>
__global__ __launch_bounds__(256, 2) void k_scored_many(ScoredAttn a) {
  using T = ManyTile<DH, MODE>;
  constexpr int TK = T::TK, ROWB = T::ROWB, DB = T::DB, KK = T::KK, CH = T::CH, RPC = T::RPC, NW = T::NW, NS = T::NS, CPW = T::CPW, LPW = T::LPW, SLOTS = T::SLOTS;
  __shared__ __align__(1024) unsigned char smem[T::LDS];
  __shared__ int red[3 * NW], red2[3 * NW];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int l32 = lane % 32, lhi = lane / 32;
  const ScoredItem item = scored_item(a, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such item
  const int nq = item.n, grp = a.H / a.Hkv;
  const int p = item.packed + min(wave * 32 + l32, nq - 1), jq = item.row + p / grp, hq = kvh * grp + p % grp;
  const uint32_t place = (uint32_t)jq * (uint32_t)a.H + (uint32_t)hq;
  const Shape sh(a);
  RowMask row;
  TileTests tests;
  int k_lo = split * item.chunk, k_hi, most;  // most: the largest limit of this wave's rows
  {
    const int i = position_of(a, PAGED, b, jq);
    row.limit = limit_of(a, b, item.keys, i);
    row.pos = i;
    if ((MODE & BIASED) && a.slopes) row.slope = sh.slope(a.slopes[hq]);
    int lo = 0x7fffffff, hi = -1;
    if constexpr (MODE & DOCS) {
      row.doc = i >= 0 && i < a.L ? a.doc[(size_t)b * a.L + i] : -1;
      if (row.doc < 0) row.limit = 0;
      lo = wave_min_i(row.doc < 0 ? 0x7fffffff : row.doc);
      hi = wave_max_i(row.doc);
      tests.one = __all(row.doc == hi);
    }
    most = wave_max_i(row.limit);
    if (lane == 0) { red2[3 * wave] = most; red2[3 * wave + 1] = lo; red2[3 * wave + 2] = hi; }
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      all = max(all, red2[3 * w]);
      lo = min(lo, red2[3 * w + 1]);
      hi = max(hi, red2[3 * w + 2]);
    }
    all = __builtin_amdgcn_readfirstlane(all);
    if constexpr (MODE & DOCS) {
      int end;
      doc_range(a.doc + (size_t)b * a.L, item.keys, lo, hi, red, &tests.first, &end, &tests.solid);
      row.limit = min(row.limit, end);  // (the sweep ends there, in the middle of a tile)
      all = min(all, end);
      k_lo = max(k_lo, tests.first / TK * TK);
    }
    tests.least = wave_min_i(row.limit);
    k_hi = min(all, (int)min((long)split * item.chunk + item.chunk, 0x7fffffffl));
    k_hi = max(k_hi, k_lo);
  }
  const int n_tiles = (k_hi - k_lo + TK - 1) / TK;
  // this wave's tiles: up to its rows' largest limit (rows that do not exist: none), the first n_clean of them without tests
  const int n_mine = wave * 32 >= nq ? 0 : min(n_tiles, max(0, (min(most, k_hi) - k_lo + TK - 1) / TK));
  const int n_clean = (MODE & DOCS) && !tests.solid ? 0 : max(0, (tests.least - k_lo) / TK);

  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>((const bf16_t *)a.q + (size_t)place * DH + lhi * 8 + kk * 16);
  floatx16 acc_o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[db][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float sc = sh.sc;

  // Stage of a tile.  (Where the first tile has keys of another document the second starts the unrolled loop, and has stage 0.)
  const int turn = (MODE == DOCS) && tests.first > k_lo ? NS - 1 : 0;
  auto stage = [&](int t) { return (uint32_t)(t + turn) % NS; };
  // Copies: copy c of a wave fills rows (c * NW + wave) * RPC and on.
  const uint32_t lds0 = lds_offset_of(smem);
  KeyPlaces<PAGED, DH> places(a, b, kvh);
  const int row0 = wave * RPC + lane / CH;  // (the rows of a wave's copies differ by 16 or lie in one half, so that they share the swizzle)
  const uint32_t off_k = (uint32_t)(row0 & 15) * places.stride + T::k_chunk(row0, lane % CH) * 16u;
  const uint32_t off_v = (uint32_t)(row0 & 15) * places.stride + T::v_chunk(row0, lane % CH) * 16u;
  static_assert(CPW == 1 || NW * RPC == 16, "");
  size_t off[2];
  auto one_copy = [&](int t, int c) {  // of a tile all of whose keys exist
    const uint32_t base = lds0 + stage(t) * T::STAGE;
    if ((MODE & DOCS) && c == 2 * CPW) {
      dma4(a.doc + (size_t)b * a.L + k_lo + t * TK + l32, base + 2 * T::REGION + wave * 256u);
      return;
    }
    const int i = c / 2;
    const size_t o = off[CPW == 1 ? wave * RPC / 16 : i];
    const uint32_t to = __builtin_amdgcn_readfirstlane(base + (c & 1) * T::REGION + (uint32_t)(i * NW + wave) * 1024u);
    if constexpr (ONCE) dma16_s_once((c & 1 ? places.v : places.k) + o, c & 1 ? off_v : off_k, to);
    else dma16_s((c & 1 ? places.v : places.k) + o, c & 1 ? off_v : off_k, to);
  };
  auto last_copies = [&](int t) {  // keys past the end are the last one again, masked later
    const uint32_t base = lds0 + stage(t) * T::STAGE;
    const int last = k_hi - 1 - (k_lo + t * TK);
#pragma unroll
    for (int i = 0; i < CPW; ++i) {
      const int to = (i * NW + wave) * RPC + lane / CH, r = min(to, last);
      const size_t o = (r >= 16 ? off[1] : off[0]) + (size_t)(r & 15) * places.stride;
      dma16(places.k + o + T::k_chunk(to, lane % CH) * 16, base + (uint32_t)(i * NW + wave) * 1024u);
      dma16(places.v + o + T::v_chunk(to, lane % CH) * 16, base + T::REGION + (uint32_t)(i * NW + wave) * 1024u);
    }
    if (MODE & DOCS) dma4(a.doc + (size_t)b * a.L + k_lo + t * TK + min(l32, last), base + 2 * T::REGION + wave * 256u);
  };
  auto full = [&](int t) { return k_lo + (t + 1) * TK <= k_hi; };
  auto next_halves = [&](int t) {  // where tile t lies, and the question for the one behind it
    places.halves(k_lo + t * TK, off);
    places.ask(k_lo + (t + 1) * TK, k_hi - 1);
  };
  auto issue = [&](int t) {
    next_halves(t);
    if (full(t)) {
#pragma unroll
      for (int c = 0; c < LPW; ++c) one_copy(t, c);
    } else {
      last_copies(t);
    }
  };
  if (n_tiles > 0) places.ask(k_lo, k_hi - 1);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < n_tiles) issue(s);
  auto landed = [&](int t) {  // tile t, of those issued so far (up to t + NS - 2)
    if (t + NS - 2 < n_tiles) wait_vmcnt<(NS - 2) * LPW>();
    else wait_vmcnt<0>();
  };
  auto landed_next = [&](int t) {  // tile t + 1, of those up to t + NS - 2
    if (t + NS - 2 < n_tiles) wait_vmcnt<(NS - 3) * LPW>();
    else wait_vmcnt<0>();
  };
  landed(0);
  __syncthreads();

  if (n_mine > 0) {
    floatx16 s_cur;
#pragma unroll
    for (int e = 0; e < 16; ++e) s_cur[e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(smem + stage(0) * T::STAGE + l32 * ROWB + T::k_chunk(l32, 2 * kk + lhi) * 16);
      s_cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], s_cur, 0, 0, 0);
    }
    // V^T and the rounded probabilities of the tile whose product is still to be issued (zero before the first)
    bf16x8 vf[2][DB], pf[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[ks][e] = (__bf16)0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[ks][db] = pf[ks];
    }
    const int vrow = 4 * lhi + (lane % 16) / 4, hb = (lane / 16) & 1;
    auto pv = [&](int ks, int db) { acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][db], pf[ks], acc_o[db], 0, 0, 0); };
    // TEST: what tile t is tested for: NOTHING (then tile t + NS - 1 exists in full), the rows' LIMITs, or ALL.  STAGE: the LDS stage of tile t where
    // it is known when compiled, else -1.
    enum { NOTHING, LIMIT, ALL };
    auto body = [&](int t, auto test_c, auto stage_c) {
      constexpr int TEST = decltype(test_c)::value;
      constexpr bool CLEAN = TEST == NOTHING;
      constexpr int STAGE = decltype(stage_c)::value;
      const int sidx = STAGE >= 0 ? STAGE : (int)stage(t);
      const bool more = CLEAN || t + NS - 1 < n_tiles, spread = CLEAN || (more && full(t + NS - 1));
      if (CLEAN) wait_vmcnt<(NS - 3) * LPW>();
      else landed_next(t);
      __syncthreads();  // tile t + 1 is in LDS; everyone is done with tile t - 1's stage
      if (more) next_halves(t + NS - 1);
      if (!CLEAN && more && !spread) last_copies(t + NS - 1);
      auto copy_behind = [&](int product) {
        constexpr int EVERY = (DB + SLOTS) / (2 * CPW);
        if (product % EVERY == EVERY / 2 && (CLEAN || spread)) one_copy(t + NS - 1, product / EVERY);
        if ((MODE & DOCS) && product == DB + SLOTS - 1 && spread) one_copy(t + NS - 1, 2 * CPW);
      };
      const unsigned char *st = smem + (size_t)sidx * T::STAGE;
      const unsigned char *st_next = smem + (size_t)((sidx + 1) % NS) * T::STAGE;
      bf16x8 kf[KK];
      auto read_k = [&](int kk) { kf[kk] = *reinterpret_cast<const bf16x8 *>(st_next + l32 * ROWB + T::k_chunk(l32, 2 * kk + lhi) * 16); };
      auto read_v = [&](int ks, int db) {
        const unsigned char *at = st + T::REGION + (vrow + 16 * ks) * ROWB + T::v_pair(vrow, db * 2 + hb) * 32 + 8 * (lane % 4);
        const shortx4 g0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at));
        const shortx4 g1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at + 8 * ROWB));
        vf[ks][db] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(g0, g1, 0, 1, 2, 3, 4, 5, 6, 7));
      };
#pragma unroll
      for (int kk = 0; kk < KK / 2; ++kk) read_k(kk);
      // Reshaping and the test of limits: behind the first products, without a branch; other tests ahead of everything.
      const int k0 = k_lo + t * TK, below = row.limit - (k0 + 4 * lhi);
      const float d0 = (float)(row.pos - (k0 + 4 * lhi));
      bool tested = TEST == LIMIT;
      if constexpr (TEST == ALL)
        tested = shape_scores<MODE>(s_cur, sh, row, tests, k0, lhi, l32, reinterpret_cast<const int32_t *>(st + 2 * T::REGION + wave * 256));
      __builtin_amdgcn_sched_barrier(0);
      float mx = -INFINITY;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        pv(0, db);
        read_k(KK / 2 + db);
        copy_behind(db);
        constexpr int PER = 16 / DB;
        if constexpr (TEST != ALL) {
#pragma unroll
          for (int e = PER * db; e < PER * (db + 1); ++e) {
            const int key = 8 * (e / 4) + (e % 4);
            if (MODE & CAPPED) s_cur[e] = sh.cap(s_cur[e]);
            if (MODE & BIASED) s_cur[e] = fmaf(-row.slope, fabsf(d0 - (float)key), s_cur[e]);
            if (TEST == LIMIT) s_cur[e] = key < below ? s_cur[e] : -INFINITY;
          }
        }
#pragma unroll
        for (int e = PER * db; e < PER * (db + 1); ++e) mx = fmaxf(mx, s_cur[e]);
        __builtin_amdgcn_sched_barrier(0);
      }
      mx = xhalf_max(mx) * sc;
      const bool need = mx > m_run + 8.0f;
      if (__any(need)) {
        // (rare after the first tiles) the accumulator changes its reference; the half of tile t - 1's probabilities whose product is still to
        // come belongs to the old one and is scaled with it.  (Rounded a second time; corr is below 2^-8, and with it what the rounding is worth.)
        const float corr = need ? __builtin_amdgcn_exp2f(m_run - mx) : 1.0f;
        m_run = need ? mx : m_run;
        l_run *= corr;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc_o[db][e] *= corr;
        const uint4 w = __builtin_bit_cast(uint4, pf[1]);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = pack_bf16(__uint_as_float(ww[q] << 16) * corr, __uint_as_float(ww[q] & 0xffff0000u) * corr);
        pf[1] = __builtin_bit_cast(bf16x8, uint4{o[0], o[1], o[2], o[3]});
      }
      const float neg_ref = (m_run == -INFINITY) ? 0.f : -m_run;
      float pe[16], ps0 = 0.f, ps1 = 0.f;
      uint32_t pw[8];
      const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3f803f80u);
      floatx16 s_next;
#pragma unroll
      for (int e = 0; e < 16; ++e) s_next[e] = 0.f;
      auto round_pair = [&](int i) {
        pw[i] = pack_bf16(pe[2 * i], pe[2 * i + 1]);
        float &ps = (i & 1) ? ps1 : ps0;
        ps = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pw[i]), ones, ps, false);
      };
      auto exps = [](int slot) { return slot < 0 ? 0 : 16 * (slot + 1) / SLOTS; };  // taken by then
#pragma unroll
      for (int slot = 0; slot < SLOTS; ++slot) {
        if (slot < DB) {
          pv(1, slot);
          read_v(0, slot);
        } else {
          s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[slot - DB], qf[slot - DB], s_next, 0, 0, 0);
          if (slot < 2 * DB) read_v(1, slot - DB);
        }
        copy_behind(DB + slot);
#pragma unroll
        for (int e = exps(slot - 1); e < exps(slot); ++e) pe[e] = __builtin_amdgcn_exp2f(fmaf(s_cur[e], sc, neg_ref));
#pragma unroll
        for (int i = exps(slot - 2) / 2; i < exps(slot - 1) / 2; ++i) round_pair(i);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = exps(SLOTS - 2) / 2; i < 8; ++i) round_pair(i);
      l_run += ps0 + ps1;  // (this lane's keys; the other half's are added behind the loop)
      pf[0] = __builtin_bit_cast(bf16x8, uint4{pw[0], pw[1], pw[2], pw[3]});
      pf[1] = __builtin_bit_cast(bf16x8, uint4{pw[4], pw[5], pw[6], pw[7]});
      if (tested) take_out_nonfinite<DB>(vf, pf, acc_o);
      s_cur = s_next;
    };
    const int n_fast = min(min(n_clean, n_mine), n_tiles - NS);  // (each with a further tile to fetch that is not the last)
    auto one = [&](int t, auto test_c) { body(t, test_c, std::integral_constant<int, -1>{}); };
    using nothing = std::integral_constant<int, NOTHING>;
    using limit = std::integral_constant<int, LIMIT>;
    using all = std::integral_constant<int, ALL>;
    int t = 0;
    if constexpr (MODE == DOCS_ANY) {
      for (; t < n_mine; ++t) one(t, all{});
    } else {
      if constexpr (MODE == DOCS) {
        const int n_all = tests.solid ? (tests.first > k_lo ? 1 : 0) : n_mine;  // (solid: the first tile may have keys of another document)
        for (; t < n_all; ++t) one(t, all{});
      }
      for (; t + NS <= n_fast; t += NS) {  // stage(t) == 0 here
        body(t, nothing{}, std::integral_constant<int, 0>{});
        body(t + 1, nothing{}, std::integral_constant<int, 1>{});
        body(t + 2, nothing{}, std::integral_constant<int, 2>{});
        body(t + 3, nothing{}, std::integral_constant<int, 3>{});
      }
      for (; t < n_mine; ++t) one(t, limit{});
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) pv(ks, db);  // the last tile's
    l_run = xhalf_sum(l_run);
  }
  // a wave that is done, or has no rows, keeps its share of the copies and meets the same barriers
  for (int t = n_mine; t < n_tiles; ++t) {
    landed_next(t);
    __syncthreads();
    if (t + NS - 1 < n_tiles) issue(t + NS - 1);
  }
  if (PAGED && places.bad && lane == 0) *a.status = a.bad_page_code;
  __syncthreads();  // every wave is done with the tiles
  const bool exists = wave * 32 + l32 < nq;
  if (a.n_split && kvh == 0 && split == 0 && lhi == 0 && exists) a.n_split[jq] = item.splits;
  if (item.splits > 1) {
    if (exists) store_scored_partial<DH>(a, acc_o, item, place, jq, lhi, m_run, l_run);
    if (a.fused) merge_splits_last<bf16_t, DH>(a, item, red, reinterpret_cast<float *>(smem));
    return;
  }
  if (wave * 32 >= nq) return;
  // whole rows leave by way of LDS: 16-byte chunk c of row r lies at c ^ (r % chunks)
  constexpr int RPI = WAVE / CH;
  unsigned char *rows = smem + wave * 32 * ROWB;
  const float inv = inverse_of(l_run);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2 *>(rows + l32 * ROWB + (((db * 4 + g) ^ (l32 % CH)) * 16) + lhi * 8) =
          uint2{pack_bf16(acc_o[db][4 * g] * inv, acc_o[db][4 * g + 1] * inv), pack_bf16(acc_o[db][4 * g + 2] * inv, acc_o[db][4 * g + 3] * inv)};
  asm volatile("" : : : "memory");  // the reads below are of another type (LDS accesses of a wave keep their order)
  const int cc = lane % CH;
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = RPI * i + lane / CH;
    const uint4 v = *reinterpret_cast<const uint4 *>(rows + r * ROWB + ((cc ^ (r % CH)) * 16));
    const uint32_t at = (uint32_t)__shfl((int)place, r, WAVE);
    if (wave * 32 + r < nq) *(reinterpret_cast<uint4 *>((bf16_t *)a.out + (size_t)at * DH) + cc) = v;
  }
}

enum class Form { FEW, MANY, ONCE };
template <Form FORM, int DH, bool PAGED, int MODE> void launch_scored(const ScoredAttn &a, hipStream_t s) {
  if constexpr (FORM == Form::FEW) k_scored_few<DH, PAGED, MODE><<<(int)scored_grid(a), 256, 0, s>>>(a);
  else k_scored_many<DH, PAGED, MODE, FORM == Form::ONCE><<<(int)scored_grid(a), 256, 0, s>>>(a);
}
template <Form FORM, bool PAGED> void launch_by_shape(const ScoredAttn &a, hipStream_t s) {
  auto go = [&](auto mode_c) {
    constexpr int MODE = decltype(mode_c)::value;
    if (a.dh == 64) launch_scored<FORM, 64, PAGED, MODE>(a, s);
    else launch_scored<FORM, 128, PAGED, MODE>(a, s);
  };
  switch (mode_of(a)) {
    case PLAIN: return go(std::integral_constant<int, PLAIN>{});
    case CAPPED: return go(std::integral_constant<int, CAPPED>{});
    case BIASED: return go(std::integral_constant<int, BIASED>{});
    case CAPPED | BIASED: return go(std::integral_constant<int, CAPPED | BIASED>{});
  }
  if constexpr (!PAGED) {
    if (mode_of(a) == DOCS) go(std::integral_constant<int, DOCS>{});
    else go(std::integral_constant<int, DOCS_ANY>{});
  }
}

}  // namespace

}  // namespace dy
