// Partial (row-sparse) attention over a key/value cache of 8-bit codes: exact attention rows of listed queries against all keys of
// their sequence, c = sum_j softmax_j(q . k_j / sqrt(dh)) v_j with k_j, v_j = code * scale.  [Sec. 3.3 salient path; Alg. 3: C_sal]
#include "attention_common.h"
#include <float.h>
#include <type_traits>

namespace dy {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// a pointer into global memory that all lanes agree on, in scalar registers
template <typename P> using Global = __attribute__((address_space(1))) P *;
template <typename P> __device__ __forceinline__ Global<P> uniform(P *p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (Global<P>)(((uint64_t)hi << 32) | lo);
}

// computed here, not where it is used (the compiler would sink it past a branch, away from the products it is to run under)
template <typename V> __device__ __forceinline__ void here(V &v) { asm volatile("" : "+v"(v)); }

// keys of sequence b
__device__ __forceinline__ int keys_of(const QuantAttn &q, int L, int b) {
  return q.kv_len ? min(max(q.kv_len[b], 0), L) : L;
}

// un-normalised rows of a split.  One without a key counts for nothing; where all are without one, the first makes the row zero
template <int DH>
__device__ __forceinline__ void store_partial(const AttnArgs &a, const floatx16 (&acc_o)[DH / 32], int split, uint32_t place, int lhi, bool none,
                                              float m_run, float l_run) {
  const size_t at = (size_t)split * a.rows.cap * a.H + place;
  float *po = a.part_o + at * DH + 4 * lhi;
#pragma unroll
  for (int db = 0; db < DH / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4 *>(po + db * 32 + 8 * g) = float4{acc_o[db][4 * g], acc_o[db][4 * g + 1], acc_o[db][4 * g + 2], acc_o[db][4 * g + 3]};
  if (lhi == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{none && split == 0 ? 0.f : m_run * LN2, none && split == 0 ? 1.f : l_run};
}

// ---- 32 packed query rows a workgroup: few rows ------------------------------------------------------------
// Bound by the codes' way from memory (one row of 8 x 32768 keys: 401 us for 2.2 GB, 5.5 TB/s) and, where several workgroups read the same
// keys, by the conversion of every code to bf16, which each repeats.  So the four waves share nothing: each streams key tiles of its own
// (tile wave, wave + 4, ..) through its own ring in LDS, with no barrier in the loop, and their results are merged once at the end.  Products
// are S^T = K Q^T and O^T = V^T P^T: a lane's scores are those of one query, so that maximum and sum need one exchange between the
// halves of the wave, and P has the layout that the second product wants.  K: a lane reads 16 codes at a time and converts them where they
// are.  V: the transposing 8-bit read gives a lane one column of eight keys.  A key's V scale is the same for all columns and joins the
// probability in fp32 ahead of its one rounding; its K scale, a power of two, joins the conversion (int8: the score).
// Two stages a wave leave room for two workgroups a CU, which hide each other's latencies: 285 rows of 16 sequences of 1280 keys at most,
// int8, 43 us; four stages and one workgroup a CU 57.
template <int DH_> struct STile {
  static constexpr int DH = DH_, NW = 4, NS = 2;
  static constexpr int BQ = 32, TK = 32;                        // query rows, keys of a wave's tile
  static constexpr int CH = DH / 16, RPC = 1024 / DH;           // 16-byte chunks of a key, keys of a copy
  static constexpr int RAW = TK * DH, COPIES = RAW / 1024;      // codes of K (and of V)
  static constexpr int STAGE = 2 * RAW + 8 * TK, PER_TILE = 2 * COPIES + 1;
  static constexpr int DB = DH / 32, KK = DH / 16, WORDS = 2 * KK;
  static constexpr int PER_WAVE = (DB * 16 + 2) * 64;           // floats of a wave's result
  static constexpr int RING = NS * STAGE, LDS = NW * RING;
  static_assert((NS - 1) * PER_TILE < 64 && (NW - 1) * PER_WAVE * 4 <= LDS, "vmcnt immediate, merge scratch");
  // position of 16-byte chunk c of row r: the rows that a read serves at a time cover all banks once
  __device__ static __forceinline__ int k_chunk(int r, int c) { return DH == 128 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3); }
  __device__ static __forceinline__ int v_chunk(int r, int c) {
    return DH == 128 ? c ^ (2 * ((r >> 1) & 1) + 4 * ((r >> 3) & 1)) : c ^ (2 * ((r >> 3) & 1));
  }
};

template <int DH, int F>
__global__ __launch_bounds__(256, 2) void k_attn_quant_stream(AttnArgs a, QuantAttn qc, int q_tiles) {
  using T = STile<DH>;
  typedef int intx2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) intx2 lds_intx2;
  constexpr int TK = T::TK, DB = T::DB, KK = T::KK, CH = T::CH, NW = T::NW, NS = T::NS, WORDS = T::WORDS;
  __shared__ __align__(1024) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int l32 = lane % 32, lhi = lane / 32;
  const AttnItem item = attn_work_item_grouped(a, T::BQ, q_tiles, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such tile
  const int nq = item.n, grp = a.H / a.Hkv;
  uint32_t place;  // row * H + head of this lane's query (rows past the end: the last one again, their results are never stored)
  {
    const int p = item.packed + min(l32, nq - 1);
    place = (uint32_t)(item.row + p / grp) * (uint32_t)a.H + (uint32_t)(kvh * grp + p % grp);
  }
  const int Lk = keys_of(qc, a.L, b);
  const int k_lo = min(split * a.chunk, Lk), k_hi = min(Lk, k_lo + a.chunk);
  const int tiles = (k_hi - k_lo + TK - 1) / TK, n_tiles = tiles > wave ? (tiles - wave + NW - 1) / NW : 0;  // this wave's: wave, wave + 4, ..

  // Copies of codes and scales, tile by tile, into the wave's own ring.
  unsigned char *own = smem + wave * T::RING;
  const uint32_t lds0 = lds_offset_of(own);
  const uint32_t stride = (uint32_t)a.Hkv * DH;
  const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH, first_s = ((size_t)b * a.Hkv + kvh) * a.L;
  const uint8_t *kc = (const uint8_t *)uniform(qc.cache.k + first), *vc = (const uint8_t *)uniform(qc.cache.v + first);
  const float *src_s = (lhi ? qc.cache.vs : qc.cache.ks) + first_s;
  uint32_t off_k[T::COPIES], off_v[T::COPIES];  // of a full tile
  auto offset = [&](int i, int last, int v) {
    const int row = i * T::RPC + lane / CH, p = lane % CH;
    return (uint32_t)min(row, last) * stride + (v ? T::v_chunk(row, p) : T::k_chunk(row, p)) * 16u;
  };
#pragma unroll
  for (int i = 0; i < T::COPIES; ++i) {
    off_k[i] = offset(i, TK - 1, 0);
    off_v[i] = offset(i, TK - 1, 1);
  }
  // full: all of the tile's keys exist; else those past the end are the last one again, masked later
  auto issue = [&](int n, auto full_c) {
    constexpr bool FULL = decltype(full_c)::value;
    const uint32_t base = lds0 + (uint32_t)(n % NS) * T::STAGE;
    const int k0 = k_lo + (wave + n * NW) * TK, last = min(k_hi - 1 - k0, TK - 1);
    const uint8_t *k = kc + (size_t)k0 * stride, *v = vc + (size_t)k0 * stride;
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
      dma16_s(k, FULL ? off_k[i] : offset(i, last, 0), base + i * 1024u);
      dma16_s(v, FULL ? off_v[i] : offset(i, last, 1), base + T::RAW + i * 1024u);
    }
    dma4(src_s + k0 + (FULL ? l32 : min(l32, last)), base + 2 * T::RAW);
  };
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < n_tiles) issue(s, std::false_type{});

  // (a lane holds the elements of the chunks that it reads of a key: those of half the head, CH / 2 neighbouring chunks)
  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>((const bf16_t *)a.q + (size_t)place * DH + lhi * (DH / 2) + kk * 8);
  floatx16 acc_o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[db][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float sc = LOG2E / sqrtf((float)DH);  // scores are kept in the log2 domain
  const int j8 = (lane % 16) / 2, hb = (lane / 16) & 1;
  const int vrow = 4 * lhi + j8 % 4 + 8 * (j8 / 4);  // (+ 16 of the second step)

  if (n_tiles > 0) {
    uint4 kr[KK / 2];   // codes of K, and the scale of this lane's key
    intx2 vr[2][DB];    // codes of V, transposed
    float kscale = 0.f;
    bf16x8 kf[KK], vf[2][DB], pf[2];
    floatx16 s_cur, s_next;
    auto stage = [&](int n) { return own + (n % NS) * T::STAGE; };
    auto read_k = [&](int n) {
      const unsigned char *st = stage(n);
#pragma unroll
      for (int i = 0; i < KK / 2; ++i) kr[i] = *reinterpret_cast<const uint4 *>(st + l32 * DH + T::k_chunk(l32, lhi * (CH / 2) + i) * 16);
      if (F == Q_E4M3) kscale = *reinterpret_cast<const float *>(st + 2 * T::RAW + 4 * l32);
    };
    auto read_v = [&](int n) {
      const unsigned char *st = stage(n);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const int row = vrow + 16 * k;
          vr[k][db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_intx2 *)(st + T::RAW + row * DH + T::v_chunk(row, 2 * db + hb) * 16 + 8 * (lane % 2)));
        }
    };
    // a word of four codes to half an operand
    auto convert_k = [&](int w) {
      const uint32_t word = w % 4 == 0 ? kr[w / 4].x : w % 4 == 1 ? kr[w / 4].y : w % 4 == 2 ? kr[w / 4].z : kr[w / 4].w;
      const uint2 r = q_bf16<F>(word, kscale);
      uint4 u = __builtin_bit_cast(uint4, kf[w / 2]);
      if (w % 2) { u.z = r.x; u.w = r.y; } else { u.x = r.x; u.y = r.y; }
      kf[w / 2] = __builtin_bit_cast(bf16x8, u);
    };
    auto convert_v = [&](int w) {
      const int k = w / (2 * DB), db = w / 2 % DB;
      const uint2 r = q_bf16<F>((uint32_t)(w % 2 ? vr[k][db].y : vr[k][db].x), 1.f);
      uint4 u = __builtin_bit_cast(uint4, vf[k][db]);
      if (w % 2) { u.z = r.x; u.w = r.y; } else { u.x = r.x; u.y = r.y; }
      vf[k][db] = __builtin_bit_cast(bf16x8, u);
    };
    auto pv = [&](int i) { acc_o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i / DB][i % DB], pf[i / DB], acc_o[i % DB], 0, 0, 0); };
    auto qk = [&](int kk) { s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], s_next, 0, 0, 0); };

    // scores of the first tile
    if (NS < n_tiles + 1) wait_vmcnt<(NS - 1) * T::PER_TILE>();
    else wait_vmcnt<0>();
    read_k(0);
#pragma unroll
    for (int e = 0; e < 16; ++e) s_next[e] = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[k][e] = (__bf16)0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[k][db] = pf[k];
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w) convert_k(w);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qk(kk);
    s_cur = s_next;

    // Tile n: P V of tile n - 1 while half of tile n's exponentials are taken and K of tile n + 1 is converted, then the scores of tile
    // n + 1 while the other half are taken and V of tile n is converted.
    auto body = [&](int n, auto steady_c) {
      constexpr bool STEADY = decltype(steady_c)::value;
      if (STEADY || n + NS - 1 < n_tiles) wait_vmcnt<(NS - 2) * T::PER_TILE>();  // tile n + 1 has landed
      else wait_vmcnt<0>();
      read_k(n + 1);  // (behind the last tile: a stage that holds none, whose scores are dropped)
      read_v(n);
      const int k0 = k_lo + (wave + n * NW) * TK;
      const unsigned char *scales = stage(n) + 2 * T::RAW + 16 * lhi;
      float vscale[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 v4 = *reinterpret_cast<const float4 *>(scales + 4 * TK + 32 * g);
        vscale[4 * g] = v4.x; vscale[4 * g + 1] = v4.y; vscale[4 * g + 2] = v4.z; vscale[4 * g + 3] = v4.w;
        if (F == Q_INT8) {
          const float4 k4 = *reinterpret_cast<const float4 *>(scales + 32 * g);
          s_cur[4 * g] *= k4.x; s_cur[4 * g + 1] *= k4.y; s_cur[4 * g + 2] *= k4.z; s_cur[4 * g + 3] *= k4.w;
        }
      }
      if (!STEADY && k0 + TK > k_hi) {  // uniform: only the last tile can hold keys past the end
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 4 * lhi + 8 * (e / 4) + (e % 4) >= k_hi) s_cur[e] = -INFINITY;
      }
      float mx = s_cur[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s_cur[e]);
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
        // the last tile's probabilities, whose products are still to come, belong to the old reference.  (They are rounded to bf16 a second time;
        // corr is below 2^-8, and with it what the rounding is worth beside the new maximum.)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 w = __builtin_bit_cast(uint4, pf[k]);
          const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
          uint32_t o[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) o[q] = pack_bf16(__uint_as_float(ww[q] << 16) * corr, __uint_as_float(ww[q] & 0xffff0000u) * corr);
          pf[k] = __builtin_bit_cast(bf16x8, uint4{o[0], o[1], o[2], o[3]});
        }
      }
      const float neg_ref = m_run == -INFINITY ? 0.f : -m_run;
      float pe[16];
      uint32_t pw[8];
      // the scale of the value joins the probability ahead of its one rounding, to the bf16 of the matrix instruction; the sum is over what there
      // was before
      auto round_pair = [&](int i) {
        l_run += pe[2 * i] + pe[2 * i + 1];
        pw[i] = pack_bf16(pe[2 * i] * vscale[2 * i], pe[2 * i + 1] * vscale[2 * i + 1]);
      };
      auto upto = [](int slot) { return slot < 0 ? 0 : 8 * (slot + 1) / KK; };  // exponentials of a phase taken by then
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int phase = 0; phase < 2; ++phase) {
        if (phase == 1) {
          if (STEADY || n + NS < n_tiles) {
            wait_lgkmcnt0();  // tile n has been read: another may come in its place
            issue(n + NS, steady_c);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) s_next[e] = 0.f;
        }
#pragma unroll
        for (int slot = 0; slot < KK; ++slot) {
          if (phase == 0) pv(slot); else qk(slot);
#pragma unroll
          for (int w = WORDS * slot / KK; w < WORDS * (slot + 1) / KK; ++w)
            if (phase == 0) convert_k(w); else convert_v(w);
#pragma unroll
          for (int g = 8 * phase + upto(slot - 1); g < 8 * phase + upto(slot); ++g) {
            pe[g] = __builtin_amdgcn_exp2f(fmaf(s_cur[g], sc, neg_ref));
            here(pe[g]);
          }
          if (slot > 0) {
#pragma unroll
            for (int i = (8 * phase + upto(slot - 2)) / 2; i < (8 * phase + upto(slot - 1)) / 2; ++i) round_pair(i);
          } else if (phase == 1) {
#pragma unroll
            for (int i = upto(KK - 2) / 2; i < 4; ++i) round_pair(i);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = (8 + upto(KK - 2)) / 2; i < 8; ++i) round_pair(i);
      pf[0] = __builtin_bit_cast(bf16x8, uint4{pw[0], pw[1], pw[2], pw[3]});
      pf[1] = __builtin_bit_cast(bf16x8, uint4{pw[4], pw[5], pw[6], pw[7]});
      s_cur = s_next;
    };
    int n = 0;
    for (; n + NS + 1 < n_tiles; ++n) body(n, std::true_type{});  // (each with a tile to copy that is not the wave's last)
    for (; n < n_tiles; ++n) body(n, std::false_type{});
#pragma unroll
    for (int i = 0; i < KK; ++i) pv(i);  // the last tile's
    l_run = xhalf_sum(l_run);
  }

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
  if (wave > 0) return;
  float M = m_run;
#pragma unroll
  for (int w = 1; w < NW; ++w) M = fmaxf(M, mg[(size_t)(w - 1) * T::PER_WAVE + (DB * 16) * 64 + lane]);
  const float Ms = (M == -INFINITY) ? 0.f : M;
  const float c0 = __builtin_amdgcn_exp2f(m_run - Ms);
  l_run *= c0;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[db][e] *= c0;
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    const float *src = mg + (size_t)(w - 1) * T::PER_WAVE + lane;
    const float cw = __builtin_amdgcn_exp2f(src[(DB * 16) * 64] - Ms);
    l_run = fmaf(src[(DB * 16 + 1) * 64], cw, l_run);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc_o[db][e] = fmaf(src[(db * 16 + e) * 64], cw, acc_o[db][e]);
  }
  if (l32 >= nq) return;
  if (a.splits > 1) {
    store_partial<DH>(a, acc_o, split, place, lhi, tiles == 0, M, l_run);
    return;
  }
  const float inv = tiles > 0 ? 1.0f / l_run : 0.f;  // (a sequence without keys: zeros)
  bf16_t *out = (bf16_t *)a.out + (size_t)place * DH + 4 * lhi;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2 *>(out + db * 32 + 8 * g) =
          uint2{pack_bf16(acc_o[db][4 * g] * inv, acc_o[db][4 * g + 1] * inv), pack_bf16(acc_o[db][4 * g + 2] * inv, acc_o[db][4 * g + 3] * inv)};
}

template <int DH> void launch_stream(const AttnArgs &a, const QuantAttn &q, hipStream_t s) {
  using T = STile<DH>;
  const int q_tiles = max_q_tiles_grouped(a, T::BQ), grid = attn_grid_grouped(a, q_tiles);
  if (q.format == Q_E4M3) k_attn_quant_stream<DH, Q_E4M3><<<grid, 256, 0, s>>>(a, q, q_tiles);
  else k_attn_quant_stream<DH, Q_INT8><<<grid, 256, 0, s>>>(a, q, q_tiles);
}

// ---- 256 packed query rows a workgroup (heads of 64: 128): many rows -------------------------------------------
// Bound by the wait of two waves a SIMD for each other: a 32-key tile holds 1024 cycles of matrix instructions a SIMD and takes about 1600, and
// no pipe is full over a launch (7766 rows of 16 x 2048 keys, 32 heads: 308 to 327 us, matrix pipes 38 % busy, vector ALU 39 %, LDS 33 %).
// A code is converted to bf16 once for all rows of the workgroup: each lane copies 16 codes of a tile straight into LDS, several tiles ahead, converts them two tiles ahead of their use and writes them to a ring of bf16 tiles that every
// wave reads, V by the transposing read.  A wave waits for its own copies alone, since it converts what it has copied; one barrier a tile.
// While the vector ALU takes the exponentials of tile t and converts tile t + 2, the matrix pipe works through P V of tile t - 1 and the
// scores of tile t + 1.  The running reference of the softmax moves only where the maximum exceeds it by 2^8, which is rare.
// All rings repeat after six tiles and the loop is unrolled by that, so that LDS addresses are constants: 5 % (345 -> 326 us for 7766 rows
// of 16 x 2048 keys, 32 heads).  Other shapes tried there: 128 rows, four waves, two workgroups a CU 317 us to 312; 64 rows a wave, keys of
// its own, 373; 64 rows a wave and shared conversion, two waves 457, four 395; a barrier every second tile 330.
template <int DH_> struct QTile {
  static constexpr int DH = DH_, NW = DH == 128 ? 8 : 4, NT = 64 * NW, BQ = 32 * NW, TK = 32;
  static constexpr int ROWB = DH * 2, ROWK = ROWB + 16;             // bytes of a converted row; of K with a gap, so that a lane's reads differ by constants
  static constexpr int HOT_K = TK * ROWK, HOT = TK * ROWB;
  static constexpr int NK = 2, NV = 3, NR = NW == 8 ? 6 : 3, CYCLE = 6;  // converted K and V, tiles of codes and their scales; all repeat after CYCLE
  static constexpr int RAW = 2 * TK * DH;                           // a tile of codes: K and V, in the order of the lanes that copy them, 16 codes a lane
  static constexpr int AT_K = 0, AT_V = NK * HOT_K, AT_RAW = AT_V + NV * HOT, AT_RS = AT_RAW + NR * RAW, AT_SC = AT_RS + NR * NW * 256, LDS = AT_SC + NV * 8 * TK;
  static constexpr int DB = DH / 32, KK = DH / 16, SLOTS = DB + KK;
  static_assert(NT * 16 == RAW && LDS <= (NW == 8 ? 160 : 80) * 1024 && BQ * ROWB <= LDS, "eight waves to a CU; the rows leave by way of the same memory");
  // 32-byte pair p of value row r: the rows that a read serves at a time cover all banks once.  (Not so the writes of converted codes, 16 bytes a
  // lane, 32 apart.  The counters show 0.14 to 0.18 of the active LDS cycles lost to conflicts; whose they are has not been tried.)
  __device__ static __forceinline__ int v_pair(int r, int p) { return DH == 128 ? p ^ (2 * (r & 3)) : p ^ (2 * ((r >> 1) & 1)); }
};

template <int DH, int F>
__global__ __launch_bounds__(QTile<DH>::NT, 2) void k_attn_quant_tile(AttnArgs a, QuantAttn qc, int q_tiles) {
  using T = QTile<DH>;
  constexpr int TK = T::TK, ROWB = T::ROWB, DB = T::DB, KK = T::KK, SLOTS = T::SLOTS, NW = T::NW;
  __shared__ __align__(1024) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int l32 = lane % 32, lhi = lane / 32;
  const AttnItem item = attn_work_item_grouped(a, T::BQ, q_tiles, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head;
  if (b < 0) return;  // uniform: no such tile
  const int nq = item.n, grp = a.H / a.Hkv;
  int jq, hq;  // this lane's query (rows past the end: the last one again, their results are never stored)
  {
    const int p = item.packed + min(wave * 32 + l32, nq - 1);
    jq = item.row + p / grp;
    hq = kvh * grp + p % grp;
  }
  const int Lk = keys_of(qc, a.L, b), n_tiles = (Lk + TK - 1) / TK;

  bf16x8 qf[KK];
  {
    const bf16_t *qp = (const bf16_t *)a.q + ((size_t)jq * a.H + hq) * DH + lhi * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(qp + kk * 16);
  }
  floatx16 acc_o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[db][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float sc = LOG2E / sqrtf((float)DH);  // scores are kept in the log2 domain

  // Copies: a wave copies 16 codes of K or of V a lane (own_v: key own_key of a tile, codes 16 own_c and on) and those keys' scales, all
  // where the same wave reads them, so that its own wait is enough.  (Heads of 128: half of the waves K, the others V; of 64: half of the lanes.)
  const uint32_t lds0 = lds_offset_of(smem);
  const size_t stride = (size_t)a.Hkv * DH;
  const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH, first_s = ((size_t)b * a.Hkv + kvh) * a.L;
  const int own_v = DH == 128 ? wave / (NW / 2) : lhi, own_8 = DH == 128 ? wave % (NW / 2) : wave;
  const int own_key = own_8 * 8 + (DH == 128 ? lane / 8 : l32 / 4), own_c = DH == 128 ? lane % 8 : lane % 4;
  const uint8_t *codes = (own_v ? qc.cache.v : qc.cache.k) + first;
  if constexpr (DH == 128) codes = (const uint8_t *)uniform(codes);
  const float *src_s = (lane & 8 ? qc.cache.vs : qc.cache.ks) + first_s;  // (8 scales of K, 8 of V, the same again)
  const int scale_key = own_8 * 8 + lane % 8;
  const uint32_t off_full = (uint32_t)own_key * (uint32_t)stride + own_c * 16u;
  // full: all of the tile's keys exist; else those past the end are the last one again, masked later
  auto issue = [&](int t, auto st_c, auto full_c) {
    constexpr int ST = decltype(st_c)::value;
    constexpr bool FULL = decltype(full_c)::value;
    const uint32_t base = lds0 + T::AT_RAW + (ST % T::NR) * T::RAW + (uint32_t)wave * 1024u;
    const int k0 = t * TK, last = Lk - 1 - k0;
    const uint32_t off = FULL ? off_full : (uint32_t)min(own_key, last) * (uint32_t)stride + own_c * 16u;
    if constexpr (DH == 128) dma16_s(codes + (size_t)k0 * stride, off, base);
    else dma16(codes + (size_t)k0 * stride + off, base);
    dma4(src_s + k0 + (FULL ? scale_key : min(scale_key, last)), lds0 + T::AT_RS + (ST % T::NR) * (NW * 256u) + wave * 256u);
  };
  auto wait_tiles = [&](auto left_c) { wait_vmcnt<decltype(left_c)::value * 2>(); };  // all but the youngest tiles have landed
  auto hot_k = [&](int st) { return smem + T::AT_K + (st % T::NK) * T::HOT_K; };
  auto hot_v = [&](int st) { return smem + T::AT_V + (st % T::NV) * T::HOT; };
  // Conversion: this lane's codes of a tile, a word of four at a time; every second word ends 16 bytes of bf16.
  uint4 raw;
  float rs;
  auto read_raw = [&](auto st_c) {
    constexpr int ST = decltype(st_c)::value;
    raw = *reinterpret_cast<const uint4 *>(smem + T::AT_RAW + (ST % T::NR) * T::RAW + wave * 1024 + lane * 16);
    rs = *reinterpret_cast<const float *>(smem + T::AT_RS + (ST % T::NR) * (NW * 256) + wave * 256 + own_v * 32 + (own_key % 8) * 4);
  };
  const int own_at = own_v ? own_key * ROWB + T::v_pair(own_key, own_c) * 32 : own_key * T::ROWK + own_c * 32;
  uint2 even{};
  auto convert = [&](int i, auto st_c) {
    constexpr int ST = decltype(st_c)::value;
    const uint2 r = q_bf16<F>(i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w, rs);
    if (i % 2 == 0) {
      even = r;
    } else {
      const int stage = own_v ? T::AT_V + (ST % T::NV) * T::HOT : T::AT_K + (ST % T::NK) * T::HOT_K;
      *reinterpret_cast<uint4 *>(smem + stage + own_at + i / 2 * 16) = uint4{even.x, even.y, r.x, r.y};
      if (F == Q_INT8 && i == 3) *reinterpret_cast<float *>(smem + T::AT_SC + (ST % T::NV) * (8 * TK) + own_v * 4 * TK + own_key * 4) = rs;
    }
  };
  auto convert_all = [&](auto st_c) {
    read_raw(st_c);
#pragma unroll
    for (int w = 0; w < 4; ++w) convert(w, st_c);
  };
  auto barrier = []() {  // (copies that are under way stay so; the wait is one that the compiler knows of)
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
  };
  constexpr int NR = T::NR;
  using part = std::false_type;
  auto first_tile = [&](auto st_c) {
    constexpr int ST = decltype(st_c)::value;
    if constexpr (ST < NR)
      if (ST < n_tiles) issue(ST, st_c, part{});
  };
  first_tile(std::integral_constant<int, 0>{});
  first_tile(std::integral_constant<int, 1>{});
  first_tile(std::integral_constant<int, 2>{});
  first_tile(std::integral_constant<int, 3>{});
  first_tile(std::integral_constant<int, 4>{});
  first_tile(std::integral_constant<int, 5>{});
  // tile t has landed, of those up to t + ahead that exist
  auto landed = [&](int t, auto ahead_c) {
    constexpr int AHEAD = decltype(ahead_c)::value;
    if (t + AHEAD < n_tiles) wait_tiles(ahead_c);
    else if (AHEAD > 2 && t + 2 < n_tiles) wait_tiles(std::integral_constant<int, 2>{});
    else wait_tiles(std::integral_constant<int, 0>{});
  };
  landed(1, std::integral_constant<int, NR - 2>{});
  if (0 < n_tiles) convert_all(std::integral_constant<int, 0>{});
  if (1 < n_tiles) convert_all(std::integral_constant<int, 1>{});
  wait_lgkmcnt0();
  if (NR < n_tiles) issue(NR, std::integral_constant<int, NR>{}, part{});
  if (NR + 1 < n_tiles) issue(NR + 1, std::integral_constant<int, NR + 1>{}, part{});
  barrier();
  const int vrow = 4 * lhi + (lane % 16) / 4, hb = (lane / 16) & 1;

  // tile t of place ST of the cycle, for t = 0 .. n - 1, as often as the cycle fits
  auto cycles = [&](int &t, int n, auto &&each) {
    for (; t < n; t += T::CYCLE) {
      each(t, std::integral_constant<int, 0>{});
      if (t + 1 < n) each(t + 1, std::integral_constant<int, 1>{});
      if (t + 2 < n) each(t + 2, std::integral_constant<int, 2>{});
      if (t + 3 < n) each(t + 3, std::integral_constant<int, 3>{});
      if (t + 4 < n) each(t + 4, std::integral_constant<int, 4>{});
      if (t + 5 < n) each(t + 5, std::integral_constant<int, 5>{});
    }
  };
  if (wave * 32 >= nq) {  // uniform: a wave without a query converts its share
    int t0 = 0;
    cycles(t0, n_tiles, [&](int t, auto st_c) {
      constexpr int ST = decltype(st_c)::value;
      landed(t + 2, std::integral_constant<int, NR - 1>{});
      barrier();
      if (t + 2 < n_tiles) convert_all(std::integral_constant<int, ST + 2>{});
      wait_lgkmcnt0();
      if (t + 2 + NR < n_tiles) issue(t + 2 + NR, std::integral_constant<int, ST + 2 + NR>{}, part{});
    });
  } else if (n_tiles > 0) {
    floatx16 s_cur;
#pragma unroll
    for (int e = 0; e < 16; ++e) s_cur[e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(hot_k(0) + l32 * T::ROWK + lhi * 16 + kk * 32);
      s_cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], s_cur, 0, 0, 0);
    }
    bf16x8 vf[2][DB], pf[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[ks][e] = (__bf16)0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[ks][db] = pf[ks];
    }
    auto pv = [&](int ks, int db) {  // O^T += V^T P^T of the tile held in vf / pf
      acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][db], pf[ks], acc_o[db], 0, 0, 0);
    };
    auto body = [&](int t, auto steady_c, auto stage_c) {
      constexpr bool STEADY = decltype(steady_c)::value;
      constexpr int ST = decltype(stage_c)::value;
      if (STEADY) wait_tiles(std::integral_constant<int, NR - 1>{});
      else landed(t + 2, std::integral_constant<int, NR - 1>{});
      barrier();  // K of tile t + 1 and V of tile t are converted
      const bool more = STEADY || t + 2 < n_tiles;
      if (more) read_raw(std::integral_constant<int, ST + 2>{});
      const unsigned char *kt = hot_k(ST + 1), *vt = hot_v(ST);
      bf16x8 kf[KK / 2];
      auto read_k = [&](int kk) { kf[kk % (KK / 2)] = *reinterpret_cast<const bf16x8 *>(kt + l32 * T::ROWK + lhi * 16 + kk * 32); };
      auto read_v = [&](int ks, int db) {
        const unsigned char *p = vt + vrow * ROWB + 8 * (lane % 4) + ks * 16 * ROWB + T::v_pair(vrow, db * 2 + hb) * 32;
        const shortx4 g0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p));
        const shortx4 g1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p + 8 * ROWB));
        vf[ks][db] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(g0, g1, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      const int k0 = t * TK;
      const unsigned char *scales = smem + T::AT_SC + (ST % T::NV) * (8 * TK) + 16 * lhi;  // (int8)
      if constexpr (F == Q_INT8) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 k4 = *reinterpret_cast<const float4 *>(scales + 32 * g);
          s_cur[4 * g] *= k4.x; s_cur[4 * g + 1] *= k4.y; s_cur[4 * g + 2] *= k4.z; s_cur[4 * g + 3] *= k4.w;
        }
      }
      if (!STEADY && k0 + TK > Lk) {  // uniform: only the last tile can hold keys past the end
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 4 * lhi + 8 * (e / 4) + (e % 4) >= Lk) s_cur[e] = -INFINITY;
      }
      auto convert_at = [&](int product) {  // behind the first three quarters of the products, so that all is written well ahead of the barrier
        constexpr int OVER = 3 * DB;
        if (more && product < OVER) {
#pragma unroll
          for (int w = product * 4 / OVER; w < (product + 1) * 4 / OVER; ++w) convert(w, std::integral_constant<int, ST + 2>{});
        }
      };
      __builtin_amdgcn_sched_barrier(0);
      float mx = s_cur[0];
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        pv(0, db);
        read_k(db);
        convert_at(db);
#pragma unroll
        for (int e = 16 / DB * db; e < 16 / DB * (db + 1); ++e) mx = fmaxf(mx, s_cur[e]);
        __builtin_amdgcn_sched_barrier(0);
      }
      mx = xhalf_max(mx) * sc;
      const bool need = mx > m_run + 8.0f;
      if (__any(need)) {
        // (rare after the first tiles) the accumulator changes its reference; the half of tile t-1's probabilities whose product is still to
        // come belongs to the old one and is scaled with it (and rounded a second time, as in the kernel above)
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
      typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
      uintx4 pw[2];
      const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3f803f80u);
      floatx16 s_next;
#pragma unroll
      for (int e = 0; e < 16; ++e) s_next[e] = 0.f;
      // Probabilities are rounded to the bf16 of the matrix instruction.  e4m3: the row sum is taken over the rounded ones, the values that
      // P V uses, two in one instruction.  int8: the scale of the value joins the probability ahead of its one rounding, and the sum is over what
      // there was before.
      auto round_pair = [&](int i) {
        float &ps = (i & 1) ? ps1 : ps0;
        uint32_t w;
        if constexpr (F == Q_E4M3) {
          w = pack_bf16(pe[2 * i], pe[2 * i + 1]);
          ps = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), ones, ps, false);
        } else {
          const float2 v2 = *reinterpret_cast<const float2 *>(scales + 4 * TK + 32 * (i / 2) + 8 * (i % 2));
          ps += pe[2 * i] + pe[2 * i + 1];
          w = pack_bf16(pe[2 * i] * v2.x, pe[2 * i + 1] * v2.y);
        }
        pw[i / 4][i % 4] = w;
      };
      auto exps = [](int slot) { return slot < 0 ? 0 : 16 * (slot + 1) / SLOTS; };  // taken by then
#pragma unroll
      for (int slot = 0; slot < SLOTS; ++slot) {
        if (slot < DB) {  // (KK is 2 DB)
          pv(1, slot);
          read_v(0, slot);
        } else {
          s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[(slot - DB) % DB], qf[slot - DB], s_next, 0, 0, 0);
          if (slot < 2 * DB) {
            read_k(slot);
            read_v(1, slot - DB);
          }
        }
        convert_at(DB + slot);
#pragma unroll
        for (int e = exps(slot - 1); e < exps(slot); ++e) {
          pe[e] = __builtin_amdgcn_exp2f(fmaf(s_cur[e], sc, neg_ref));
          here(pe[e]);
        }
#pragma unroll
        for (int i = exps(slot - 2) / 2; i < exps(slot - 1) / 2; ++i) round_pair(i);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = exps(SLOTS - 2) / 2; i < 8; ++i) round_pair(i);
      if (STEADY || t + 2 + NR < n_tiles) issue(t + 2 + NR, std::integral_constant<int, ST + 2 + NR>{}, steady_c);  // (the codes that lay there have been converted)
      l_run += ps0 + ps1;  // (this lane's keys; the other half's are added behind the loop)
      pf[0] = __builtin_bit_cast(bf16x8, pw[0]);
      pf[1] = __builtin_bit_cast(bf16x8, pw[1]);
      s_cur = s_next;
    };
    {
      int t = 0;
      for (; t + T::CYCLE + 2 + NR < n_tiles; t += T::CYCLE) {  // (each with a tile to copy that is not the last)
        body(t, std::true_type{}, std::integral_constant<int, 0>{});
        body(t + 1, std::true_type{}, std::integral_constant<int, 1>{});
        body(t + 2, std::true_type{}, std::integral_constant<int, 2>{});
        body(t + 3, std::true_type{}, std::integral_constant<int, 3>{});
        body(t + 4, std::true_type{}, std::integral_constant<int, 4>{});
        body(t + 5, std::true_type{}, std::integral_constant<int, 5>{});
      }
      cycles(t, n_tiles, [&](int u, auto st_c) { body(u, std::false_type{}, st_c); });
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) pv(ks, db);  // the last tile's
    l_run = xhalf_sum(l_run);
  }
  __syncthreads();  // every wave is done with the tiles
  if (wave * 32 >= nq) return;
  // whole rows leave by way of LDS: 16-byte chunk c of row r lies at c ^ (r % chunks)
  constexpr int CH = DH / 8, RPI = WAVE / CH;
  unsigned char *rows = smem + wave * 32 * ROWB;
  const float inv = n_tiles > 0 ? 1.0f / l_run : 0.f;  // (a sequence without keys: zeros)
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2 *>(rows + l32 * ROWB + (((db * 4 + g) ^ (l32 % CH)) * 16) + lhi * 8) =
          uint2{pack_bf16(acc_o[db][4 * g] * inv, acc_o[db][4 * g + 1] * inv), pack_bf16(acc_o[db][4 * g + 2] * inv, acc_o[db][4 * g + 3] * inv)};
  asm volatile("" : : : "memory");  // the reads below are of another type (LDS accesses of a wave keep their order)
  const uint32_t place = (uint32_t)jq * (uint32_t)a.H + (uint32_t)hq;
  const int cc = lane % CH;
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = RPI * i + lane / CH;
    const uint4 v = *reinterpret_cast<const uint4 *>(rows + r * ROWB + ((cc ^ (r % CH)) * 16));
    const uint32_t at = (uint32_t)__shfl((int)place, r, WAVE);
    if (wave * 32 + r < nq) *(reinterpret_cast<uint4 *>((bf16_t *)a.out + (size_t)at * DH) + cc) = v;
  }
}

template <int DH> void launch_tile(const AttnArgs &a, const QuantAttn &q, hipStream_t s) {
  using T = QTile<DH>;
  const int q_tiles = max_q_tiles_grouped(a, T::BQ), grid = attn_grid_grouped(a, q_tiles);
  if (q.format == Q_E4M3) k_attn_quant_tile<DH, Q_E4M3><<<grid, T::NT, 0, s>>>(a, q, q_tiles);
  else k_attn_quant_tile<DH, Q_INT8><<<grid, T::NT, 0, s>>>(a, q, q_tiles);
}

// ---- merge of the splits: a wave to a (row, head), its lanes the splits' weights, then the columns -------------
// Bound by the latency of its two dependent reads: 4 us for 32 (row, head) pairs of 8 splits.
constexpr int MAX_SPLITS = 128;
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_quant_merge(AttnArgs a) {
  constexpr int V = DH / WAVE;
  const int n = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap, lane = threadIdx.x % WAVE;
  const uint32_t items = (uint32_t)n * (uint32_t)a.H;
  const size_t step = (size_t)a.rows.cap * a.H;
  for (uint32_t it = blockIdx.x * 4 + threadIdx.x / WAVE; it < items; it += gridDim.x * 4) {
    float m[2], l[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int s = lane + u * WAVE;
      const float2 ml = s < a.splits ? *reinterpret_cast<const float2 *>(a.part_ml + ((size_t)s * step + it) * 2) : float2{-INFINITY, 0.f};
      m[u] = ml.x; l[u] = ml.y;
    }
    // (as in the kernels before: a maximum that is no number leaves the weights so)
    const float M = wave_max(fmaxf(m[0], m[1])), ref = M == -INFINITY ? 0.f : M;
    float w[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) w[u] = __expf(m[u] - ref);
    const float total = wave_sum(l[0] * w[0] + l[1] * w[1]);
    float o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = 0.f;
    const float *po = a.part_o + (size_t)it * DH + lane * V;
    auto weight = [&](int s) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s < WAVE ? w[0] : w[1]), s % WAVE)); };
    for (int s0 = 0; s0 < a.splits; s0 += 8) {  // (eight loads in flight; past the end the last split again, with no weight)
      float x[8][V];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][e] = po[(size_t)min(s0 + i, a.splits - 1) * step * DH + e];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float ws = s0 + i < a.splits ? weight(s0 + i) : 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(x[i][e], ws, o[e]);
      }
    }
    const float inv = 1.0f / total;
    T *out = (T *)a.out + (size_t)it * DH + lane * V;
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = from_f<T>(o[e] * inv);
  }
}

template <typename T> void launch_merge(const AttnArgs &a, hipStream_t s) {
  const long blocks = ((long)a.rows.cap * a.H + 3) / 4;
  const int grid = (int)(blocks > 8192 ? 8192 : blocks);
  if (a.dh == 64) k_quant_merge<T, 64><<<grid, 256, 0, s>>>(a);
  else k_quant_merge<T, 128><<<grid, 256, 0, s>>>(a);
}

// ---- fp32 queries and results: R packed rows a workgroup ------------------------------------------------------
// dh / 16 lanes take a key, a lane 16 of its codes, and 64 / (dh / 16) keys go through a wave at a time, each group of lanes with a running
// maximum, sum and result of its own; four waves take such steps in turn.  A lane keeps its 16 elements of the R queries and results in
// registers, so that the loop has no LDS and no barrier: per key and row 16 products and two or three moves between neighbouring lanes for
// the score, 16 for the result, every one in fp32; the scales join the score and the probability.  Groups and waves are merged at the end.
// Bound by the vector ALU (R = 2: 3882 rows of 16 x 1024 keys, 32 heads of 128, 1.63 ms, 40 TFLOP/s) or by the codes' way from memory and
// the launches (R = 1: one row of 2048 keys, 32 heads, 10.5 us).  R = 4, whose registers leave two waves a SIMD: 1.65 ms, 15.8 us.
template <int DH, int F, int R>
__global__ __launch_bounds__(256, 3) void k_attn_quant_f32(AttnArgs a, QuantAttn qc, int q_tiles) {
  constexpr int CPK = DH / 16, KS = WAVE / CPK, NW = 4, U = 2;  // lanes of a key, keys of a wave's step, waves, steps in flight
  __shared__ float part[NW][R][DH], part_ml[NW][R][2];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int c = lane % CPK, group = lane / CPK;
  const AttnItem item = attn_work_item_grouped(a, R, q_tiles, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such tile
  const int nq = item.n, grp = a.H / a.Hkv;
  auto place = [&](int r) {  // row * H + head of packed row r
    const int p = item.packed + r;
    return (uint32_t)(item.row + p / grp) * (uint32_t)a.H + (uint32_t)(kvh * grp + p % grp);
  };
  const int Lk = keys_of(qc, a.L, b);
  const int k_lo = min(split * a.chunk, Lk), k_hi = min(Lk, k_lo + a.chunk);
  const size_t stride = (size_t)a.Hkv * DH;
  const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH + c * 16, first_s = ((size_t)b * a.Hkv + kvh) * a.L;
  const uint8_t *kc = qc.cache.k + first, *vc = qc.cache.v + first;
  const float *ks = qc.cache.ks + first_s, *vs = qc.cache.vs + first_s;
  float q[R][16], acc[R][16], m_run[R], l_run[R];
  const float sc = LOG2E / sqrtf((float)DH);  // scores are kept in the log2 domain
#pragma unroll
  for (int r = 0; r < R; ++r) {  // (rows past the end: the last one again, their results are never stored)
    const float4 *src = reinterpret_cast<const float4 *>((const float *)a.q + (size_t)place(min(r, nq - 1)) * DH + c * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = src[i];
      q[r][4 * i] = x.x * sc; q[r][4 * i + 1] = x.y * sc; q[r][4 * i + 2] = x.z * sc; q[r][4 * i + 3] = x.w * sc;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[r][e] = 0.f;
    m_run[r] = -FLT_MAX;  // (finite, so that a score of -inf has the probability 0)
    l_run[r] = 0.f;
  }
  struct Step { uint4 k, v; float ks, vs; };
  auto key_of = [&](int n) { return k_lo + (n * NW + wave) * KS + group; };
  auto load = [&](int n, Step &s) {  // (keys past the end: the last one again, masked later)
    const int key = min(key_of(n), k_hi - 1);
    s.k = *reinterpret_cast<const uint4 *>(kc + (size_t)key * stride);
    s.v = *reinterpret_cast<const uint4 *>(vc + (size_t)key * stride);
    s.ks = ks[key];
    s.vs = vs[key];
  };
  auto values = [](const uint4 &w, float *x) {
    q_values<F>(w.x, 1.f, x); q_values<F>(w.y, 1.f, x + 4); q_values<F>(w.z, 1.f, x + 8); q_values<F>(w.w, 1.f, x + 12);
  };
  const int n_steps = (k_hi - k_lo + NW * KS - 1) / (NW * KS);
  Step next[U];
  if (n_steps > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) load(u, next[u]);
  }
  for (int n = 0; n < n_steps; n += U) {
    Step now[U];
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = next[u];
    if (n + U < n_steps) {
#pragma unroll
      for (int u = 0; u < U; ++u) load(n + U + u, next[u]);
    }
    float score[U][R];
    bool need = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[16];
      values(now[u].k, x);
      const bool exists = key_of(n + u) < k_hi;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float d0 = 0.f, d1 = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          d0 = fmaf(q[r][e], x[e], d0);
          d1 = fmaf(q[r][e + 1], x[e + 1], d1);
        }
        score[u][r] = exists ? lanes_sum<CPK>(d0 + d1) * now[u].ks : -INFINITY;
        need = need || score[u][r] > m_run[r] + 8.0f;
      }
    }
    if (__any(need)) {  // the running reference moves where a score exceeds it by more than 2^8: rare after the first steps
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = m_run[r];
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, score[u][r]);
        const float corr = __builtin_amdgcn_exp2f(m_run[r] - top);
        m_run[r] = top;
        l_run[r] *= corr;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][e] *= corr;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[16];
      values(now[u].v, x);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float p = __builtin_amdgcn_exp2f(score[u][r] - m_run[r]);
        l_run[r] += p;
        const float pv = p * now[u].vs;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][e] = fmaf(pv, x[e], acc[r][e]);
      }
    }
  }
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
  const bool none = k_lo >= k_hi, whole = a.splits == 1;
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
    const size_t at = place(r) + (whole ? 0 : (size_t)split * a.rows.cap * a.H);
    if (whole) {
      ((float *)a.out)[at * DH + col] = none ? 0.f : o / l;
    } else {  // (a split without keys counts for nothing; where all are without, the first makes the row zero)
      a.part_o[at * DH + col] = o;
      if (col == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{none && split == 0 ? 0.f : none ? -INFINITY : top * LN2, none && split == 0 ? 1.f : l};
    }
  }
}

template <int DH, int R> void launch_f32(const AttnArgs &a, const QuantAttn &q, hipStream_t s) {
  const int q_tiles = max_q_tiles_grouped(a, R), grid = attn_grid_grouped(a, q_tiles);
  if (q.format == Q_E4M3) k_attn_quant_f32<DH, Q_E4M3, R><<<grid, 256, 0, s>>>(a, q, q_tiles);
  else k_attn_quant_f32<DH, Q_INT8, R><<<grid, 256, 0, s>>>(a, q, q_tiles);
}

}  // namespace

// Query tile and key splits, of what the host knows: the list's capacity stands for its count, so a list with room for far more than it holds
// may get the tall form and no splits: one row of 32768 keys, 32 heads, in a list of one entry 51 us, of 32768 476.
// The prices are fits to timed launches (heads of 128, e4m3 and int8 within 10 %), ns of a workgroup per key:
//   32 rows a workgroup   7 while each CU has one; 15.5 for the 512 that the chip holds, and so on in proportion
//   256 rows              28.5 for the 256 that the chip holds (heads of 64: 128 rows, 25, 512 of them; the 32-row form 5 and 8.5)
// so 32 rows a workgroup are taken for few rows or few sequences.  32 / 256 rows, us: 285 rows of 16 sequences, 1280 keys at most,
// 45.6 / 71.3; 1941 rows 105 / 81; 1554 rows of 16 x 2048 keys 125 / 112; 102 rows of one sequence of 1024 13.5 / 24.5; 28 heads over 4,
// 1137 rows of 13 x 1277 48.3 / 50.3; heads of 64 over 2, 7764 rows of 16 x 2048 78 / 55.
// fp32: 1 row a workgroup 7 alone and 17 for 1000 of them (heads of 64: 3.7 and 9.2), 2 rows 11 and 26 (5.2 and 13).  1 / 2 rows: 3882 rows
// of 16 x 1024, 32 heads of 128, 2155 / 1632; 379 of 4 x 1024 249 / 167; 1 of 2048 10.5 / 12.2; heads of 64 over 4, 7580 rows of 16 x 2000
// 558 / 400, 45 of 16 x 1500 11.9 / 15.
// Splits pay a second launch and the partial results' way through memory, so only fp32 and the 32-row form have them, where a few workgroups
// would read long sequences: 1 row of 32768 keys, 4 heads, 1 / 8 / 32 / 128 splits 183 / 33.6 / 19.5 / 25.2 us; one row in each of 16
// sequences of 2048, 1 / 4 / 16 22.7 / 18.0 / 23.5; 102 rows of 1024, 32 heads, 1 / 2 13.5 / 16.7; fp32, heads of 64, 1 row of 32000,
// 1 / 8 / 32 / 128 120 / 22.8 / 13.5 / 17.6.
void attention_quant_plan(DType t, size_t part_elems, AttnArgs *a) {
  const long grp = a->H / a->Hkv, rows = a->offsets ? ((long)a->rows.cap + a->B - 1) / a->B : a->L, packed = rows * grp;
  const bool d128 = a->dh == 128;
  auto tiles = [&](int bq) { return (double)a->B * a->Hkv * ((packed + bq - 1) / bq); };
  struct Price { double alone, each; };  // ns a key: of one workgroup, and that each adds where there are many
  auto price_of = [&](int bq) {
    if (t == F32) return bq == 1 ? (d128 ? Price{7, 0.017} : Price{3.7, 0.0092}) : (d128 ? Price{11, 0.026} : Price{5.2, 0.013});
    if (bq == 32) return d128 ? Price{7, 15.5 / 512} : Price{5, 8.5 / 512};
    return d128 ? Price{28.5, 28.5 / 256} : Price{25, 25.0 / 512};
  };
  auto price = [&](int bq, double n) {
    const Price p = price_of(bq);
    return n * p.each > p.alone ? n * p.each : p.alone;
  };
  const int low = t == F32 ? 1 : 32, tall = t == F32 ? 2 : d128 ? 256 : 128;
  a->bq = price(tall, tiles(tall)) < price(low, tiles(low)) ? tall : low;
  a->splits = 1;
  const int BK = t == F32 ? 4096 / a->dh : 128;  // keys that the waves of a workgroup take at a time
  if (t == F32 || a->bq == 32) {
    const double n = tiles(a->bq);
    const size_t per_split = (size_t)a->rows.cap * a->H * a->dh;
    double best = 0;
    for (int s = 1; s <= MAX_SPLITS && (long)(s - 1) * BK < a->L && (s == 1 || s * per_split <= part_elems); ++s) {
      const double ns = a->L / (double)s * price(a->bq, n * s) + (s > 1 ? 3500 + 150.0 * s + 8.0 * s * per_split / 4000 : 0);
      if (s == 1 || ns < best) {
        best = ns;
        a->splits = s;
      }
    }
  }
  a->chunk = split_chunk(a->L, a->splits, BK);
  a->splits = (a->L + a->chunk - 1) / a->chunk;  // drops splits that would be empty
}

void launch_attention_quant(DType t, const AttnArgs &a, const QuantAttn &q, hipStream_t s) {
  if (a.rows.cap <= 0) return;
  if (t == F32) {
    if (a.dh == 64 && a.bq == 1) launch_f32<64, 1>(a, q, s);
    else if (a.dh == 64) launch_f32<64, 2>(a, q, s);
    else if (a.bq == 1) launch_f32<128, 1>(a, q, s);
    else launch_f32<128, 2>(a, q, s);
    if (a.splits > 1) launch_merge<float>(a, s);
    return;
  }
  if (a.bq == 32) {
    if (a.dh == 64) launch_stream<64>(a, q, s);
    else launch_stream<128>(a, q, s);
  } else {
    if (a.dh == 64) launch_tile<64>(a, q, s);
    else launch_tile<128>(a, q, s);
  }
  if (a.splits > 1) launch_merge<bf16_t>(a, s);
}

}  // namespace dy
