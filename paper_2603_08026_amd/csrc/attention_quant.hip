// Partial (row-sparse) attention over a key/value cache of 8-bit codes: exact attention rows of listed queries against all keys of
// their sequence, c = sum_j softmax_j(q . k_j / sqrt(dh)) v_j with k_j, v_j = code * scale.  [Sec. 3.3 salient path; Alg. 3: C_sal]
#include "attention_common.h"
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

// keys of sequence b
__device__ __forceinline__ int keys_of(const QuantAttn &q, int L, int b) {
  return q.kv_len ? min(max(q.kv_len[b], 0), L) : L;
}

template <int DH_, int WQ_, int WK_> struct QTile {
  static constexpr int DH = DH_, WQ = WQ_, WK = WK_, NW = WQ * WK, NT = 64 * NW;
  static constexpr int BQ = 32 * WQ, TK = 32 * WK;
  static constexpr int ROWB = DH * 2, REGION = TK * ROWB;
  static constexpr int DB = DH / 32, KK = DH / 16, CH = DH / 16;  // CH: 16-byte chunks of codes in a key
  static constexpr int PER = 2 * TK * CH / NT;                    // chunks per thread and tile
  static constexpr int PER_WAVE = (DB * 16 + 2) * 64;
  static constexpr int MERGE_BYTES = (WK - 1) * WQ * PER_WAVE * 4;
  static constexpr int LDS = 2 * REGION > MERGE_BYTES ? 2 * REGION : MERGE_BYTES;
  static_assert(PER >= 1 && PER * NT == 2 * TK * CH, "a tile is copied in whole chunks per thread");
  // 16-byte chunk c of key row r, and 32-byte pair p of value row r, in a row of the stage
  __device__ static __forceinline__ int k_chunk(int r, int c) { return DH == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7); }
  __device__ static __forceinline__ int v_pair(int r, int p) { return DH == 128 ? p ^ (2 * (r & 3)) : p ^ (2 * ((r >> 1) & 1)); }
};

template <int DH, int WQ, int WK, int F>
__global__ __launch_bounds__(64 * WQ * WK) void k_attn_quant(AttnArgs a, QuantAttn qc, int q_tiles) {
  using T = QTile<DH, WQ, WK>;
  constexpr int TK = T::TK, ROWB = T::ROWB, DB = T::DB, KK = T::KK, CH = T::CH, PER = T::PER, NT = T::NT;
  __shared__ __align__(1024) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int l32 = lane % 32, lhi = lane / 32;
  const int wq = wave / WK, wk = wave % WK;
  const AttnItem item = attn_work_item_grouped(a, T::BQ, q_tiles, blockIdx.x);
  const int b = item.seq, kvh = item.kv_head, split = item.split;
  if (b < 0) return;  // uniform: no such tile
  const int nq = item.n, grp = a.H / a.Hkv;
  int jq, hq;
  {
    int r = wq * 32 + l32;
    r = r < nq ? r : nq - 1;
    const int p = item.packed + r;
    jq = item.row + p / grp;
    hq = kvh * grp + p % grp;
  }
  const int Lk = keys_of(qc, a.L, b);
  const int k_lo = min(split * a.chunk, Lk), k_hi = min(Lk, k_lo + a.chunk);

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
  const float sc = LOG2E / sqrtf((float)DH);

  const size_t stride = (size_t)a.Hkv * DH;
  const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH, first_s = ((size_t)b * a.Hkv + kvh) * a.L;
  uint4 raw[PER];
  float scale[PER];
  auto load = [&](int k0) {  // (keys past the end: the last one again, masked later)
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int i = tid + NT * u, isv = i / (TK * CH), in = i % (TK * CH);
      const int key = min(k0 + in / CH, k_hi - 1);
      raw[u] = *reinterpret_cast<const uint4 *>((isv ? qc.cache.v : qc.cache.k) + first + (size_t)key * stride + (in % CH) * 16);
      scale[u] = (isv ? qc.cache.vs : qc.cache.ks)[first_s + key];
    }
  };
  auto store = [&]() {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int i = tid + NT * u, isv = i / (TK * CH), in = i % (TK * CH);
      const int key = in / CH, c = in % CH;
      const uint2 w0 = q_bf16<F>(raw[u].x, scale[u]), w1 = q_bf16<F>(raw[u].y, scale[u]);
      const uint2 w2 = q_bf16<F>(raw[u].z, scale[u]), w3 = q_bf16<F>(raw[u].w, scale[u]);
      unsigned char *row = smem + (isv ? T::REGION : 0) + key * ROWB;
      const int c0 = isv ? 2 * T::v_pair(key, c) : T::k_chunk(key, 2 * c), c1 = isv ? c0 + 1 : T::k_chunk(key, 2 * c + 1);
      *reinterpret_cast<uint4 *>(row + c0 * 16) = uint4{w0.x, w0.y, w1.x, w1.y};
      *reinterpret_cast<uint4 *>(row + c1 * 16) = uint4{w2.x, w2.y, w3.x, w3.y};
    }
  };

  const int krow = wk * 32 + l32;
  const int vrow = wk * 32 + 4 * lhi + (lane % 16) / 4, hb = (lane / 16) & 1;
  if (k_lo < k_hi) load(k_lo);
  for (int k0 = k_lo; k0 < k_hi; k0 += TK) {
    __syncthreads();
    store();
    __syncthreads();
    if (k0 + TK < k_hi) load(k0 + TK);
    floatx16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(smem + krow * ROWB + T::k_chunk(krow, 2 * kk + lhi) * 16);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], s, 0, 0, 0);
    }
    if (k0 + TK > k_hi) {  // uniform
      const int key_base = k0 + wk * 32 + 4 * lhi;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (key_base + 8 * (e / 4) + (e % 4) >= k_hi) s[e] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = xhalf_max(mx) * sc;
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
    const float neg_ref = (m_run == -INFINITY) ? 0.f : -m_run;
    uint32_t pw[8];
    float ps = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e], sc, neg_ref));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(s[e + 1], sc, neg_ref));
      const uint32_t w = pack_bf16(p0, p1);
      ps += __uint_as_float(w << 16) + __uint_as_float(w & 0xffff0000u);
      pw[e >> 1] = w;
    }
    l_run += xhalf_sum(ps);
    const bf16x8 pf[2] = {__builtin_bit_cast(bf16x8, uint4{pw[0], pw[1], pw[2], pw[3]}),
                          __builtin_bit_cast(bf16x8, uint4{pw[4], pw[5], pw[6], pw[7]})};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int row = vrow + ks * 16;
        const unsigned char *p = smem + T::REGION + row * ROWB + 8 * (lane % 4) + T::v_pair(row, db * 2 + hb) * 32;
        const shortx4 g0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p));
        const shortx4 g1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p + 8 * ROWB));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(g0, g1, 0, 1, 2, 3, 4, 5, 6, 7));
        acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[ks], acc_o[db], 0, 0, 0);
      }
  }

  // merge the wave columns of each query block through LDS
  if constexpr (WK > 1) {
    float *mg = reinterpret_cast<float *>(smem);
    __syncthreads();
    if (wk > 0) {
      float *dst = mg + (size_t)((wk - 1) * WQ + wq) * T::PER_WAVE + lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) dst[(db * 16 + e) * 64] = acc_o[db][e];
      dst[(DB * 16) * 64] = m_run;
      dst[(DB * 16 + 1) * 64] = l_run;
    }
    __syncthreads();
    if (wk > 0) return;
    float M = m_run;
#pragma unroll
    for (int w = 1; w < WK; ++w) M = fmaxf(M, mg[(size_t)((w - 1) * WQ + wq) * T::PER_WAVE + (DB * 16) * 64 + lane]);
    const float Ms = (M == -INFINITY) ? 0.f : M;
    const float c0 = __builtin_amdgcn_exp2f(m_run - Ms);
    l_run *= c0;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc_o[db][e] *= c0;
#pragma unroll
    for (int w = 1; w < WK; ++w) {
      const float *src = mg + (size_t)((w - 1) * WQ + wq) * T::PER_WAVE + lane;
      const float cw = __builtin_amdgcn_exp2f(src[(DB * 16) * 64] - Ms);
      l_run = fmaf(src[(DB * 16 + 1) * 64], cw, l_run);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc_o[db][e] = fmaf(src[(db * 16 + e) * 64], cw, acc_o[db][e]);
    }
    m_run = M;
  }
  if (wq * 32 + l32 >= nq) return;
  if (a.splits == 1) {
    const float inv = k_lo < k_hi ? 1.0f / l_run : 0.f;  // (a sequence without keys: zeros)
    bf16_t *out = (bf16_t *)a.out + ((size_t)jq * a.H + hq) * DH + 4 * lhi;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2 *>(out + db * 32 + 8 * g) =
            uint2{pack_bf16(acc_o[db][4 * g] * inv, acc_o[db][4 * g + 1] * inv), pack_bf16(acc_o[db][4 * g + 2] * inv, acc_o[db][4 * g + 3] * inv)};
  } else {
    const size_t at = ((size_t)split * a.rows.cap + jq) * a.H + hq;
    float *po = a.part_o + at * DH + 4 * lhi;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4 *>(po + db * 32 + 8 * g) = float4{acc_o[db][4 * g], acc_o[db][4 * g + 1], acc_o[db][4 * g + 2], acc_o[db][4 * g + 3]};
    // a split without a key counts for nothing; where all are without one, the first makes the row zero
    if (lhi == 0) {
      const bool none = k_lo >= k_hi;
      *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{none && split == 0 ? 0.f : m_run * LN2, none && split == 0 ? 1.f : l_run};
    }
  }
}

template <int DH, int WQ, int WK> void launch_tile(const AttnArgs &a, const QuantAttn &q, hipStream_t s) {
  using T = QTile<DH, WQ, WK>;
  const int q_tiles = max_q_tiles_grouped(a, T::BQ), grid = attn_grid_grouped(a, q_tiles);
  if (q.format == Q_E4M3) k_attn_quant<DH, WQ, WK, Q_E4M3><<<grid, T::NT, 0, s>>>(a, q, q_tiles);
  else k_attn_quant<DH, WQ, WK, Q_INT8><<<grid, T::NT, 0, s>>>(a, q, q_tiles);
}

// fp32 queries and results: 16 rows x 16 lanes a workgroup, tiles of 32 keys; codes become fp32 values on their way into LDS.
template <int DH, int F>
__global__ __launch_bounds__(256) void k_attn_quant_f32(AttnArgs a, QuantAttn qc) {
  typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;
  constexpr int BQ = 16, BK = 32, NT = 256, STR = DH + 4, CH = DH / 16, LD = (2 * BK * CH + NT - 1) / NT, OC = DH / 64;
  __shared__ __align__(16) float Qs[BQ][STR];
  __shared__ __align__(16) float Ks[BK][STR];
  __shared__ __align__(16) float Vs[BK][DH];
  __shared__ __align__(16) float Ps[BQ][BK + 4];
  __shared__ int tile_info[3];
  const int tid = threadIdx.x;
  if (tid == 0) find_tile(a, BQ, blockIdx.x, tile_info);
  __syncthreads();
  const int b = tile_info[0];
  if (b < 0) return;  // uniform: no such tile
  const int j0 = tile_info[1], nq = tile_info[2];
  const int h = blockIdx.y, kvh = h / (a.H / a.Hkv), split = blockIdx.z;
  const int Lk = keys_of(qc, a.L, b);
  const int k_lo = min(split * a.chunk, Lk), k_hi = min(Lk, k_lo + a.chunk);
  const size_t stride = (size_t)a.Hkv * DH;
  const size_t first = ((size_t)b * a.L * a.Hkv + kvh) * DH, first_s = ((size_t)b * a.Hkv + kvh) * a.L;
  const float by = 1.0f / sqrtf((float)DH);
  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  uint4 raw[LD];
  float scale[LD];
  auto load = [&](int k0) {  // (keys past the end: the last one again, masked later)
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int i = min(tid + NT * u, 2 * BK * CH - 1), isv = i / (BK * CH), in = i % (BK * CH);
      const int key = min(k0 + in / CH, k_hi - 1);
      raw[u] = *reinterpret_cast<const uint4 *>((isv ? qc.cache.v : qc.cache.k) + first + (size_t)key * stride + (in % CH) * 16);
      scale[u] = (isv ? qc.cache.vs : qc.cache.ks)[first_s + key];
    }
  };
  if (k_lo < k_hi) load(k_lo);
  for (int e = tid; e < BQ * DH / 4; e += NT) {
    const int r = e / (DH / 4), c = (e % (DH / 4)) * 4;
    *reinterpret_cast<floatx4 *>(&Qs[r][c]) = r < nq ? *reinterpret_cast<const floatx4 *>((const float *)a.q + ((size_t)(j0 + r) * a.H + h) * DH + c) * by : zero;
  }
  const int row = tid / 16, sub = tid % 16;
  floatx4 o[OC];
#pragma unroll
  for (int i = 0; i < OC; ++i) o[i] = zero;
  float m_run = -INFINITY, l_run = 0.f;
  for (int k0 = k_lo; k0 < k_hi; k0 += BK) {
    __syncthreads();  // previous tile fully consumed (also orders the Qs fill)
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int i = tid + NT * u;
      if (i < 2 * BK * CH) {
        const int isv = i / (BK * CH), in = i % (BK * CH), key = in / CH, c = (in % CH) * 16;
        float *dst = isv ? &Vs[key][c] : &Ks[key][c];
        q_values<F>(raw[u].x, scale[u], dst);
        q_values<F>(raw[u].y, scale[u], dst + 4);
        q_values<F>(raw[u].z, scale[u], dst + 8);
        q_values<F>(raw[u].w, scale[u], dst + 12);
      }
    }
    __syncthreads();
    if (k0 + BK < k_hi) load(k0 + BK);
    floatx4 a0 = zero, a1 = zero;
#pragma unroll
    for (int e = 0; e < DH; e += 4) {
      const floatx4 qv = *reinterpret_cast<const floatx4 *>(&Qs[row][e]);
      a0 += qv * *reinterpret_cast<const floatx4 *>(&Ks[sub][e]);
      a1 += qv * *reinterpret_cast<const floatx4 *>(&Ks[sub + 16][e]);
    }
    float s0 = (a0[0] + a0[1]) + (a0[2] + a0[3]), s1 = (a1[0] + a1[1]) + (a1[2] + a1[3]);
    if (k0 + sub >= k_hi) s0 = -INFINITY;
    if (k0 + sub + 16 >= k_hi) s1 = -INFINITY;
    float mt = fmaxf(s0, s1);
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) mt = fmaxf(mt, __shfl_xor(mt, off, 16));
    const float m_new = fmaxf(m_run, mt);  // finite: every tile holds at least one valid key
    const float corr = __expf(m_run - m_new);
    const float p0 = __expf(s0 - m_new), p1 = __expf(s1 - m_new);
    float ps = p0 + p1;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) ps += __shfl_xor(ps, off, 16);
    l_run = l_run * corr + ps;
    m_run = m_new;
    Ps[row][sub] = p0;
    Ps[row][sub + 16] = p1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < OC; ++i) o[i] *= corr;
#pragma unroll
    for (int kk = 0; kk < BK; kk += 4) {
      const floatx4 p = *reinterpret_cast<const floatx4 *>(&Ps[row][kk]);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < OC; ++i) o[i] += p[x] * *reinterpret_cast<const floatx4 *>(&Vs[kk + x][64 * i + 4 * sub]);
    }
  }
  if (row >= nq) return;
  const bool none = k_lo >= k_hi, whole = a.splits == 1;
  const size_t at = (((size_t)(whole ? 0 : split) * a.rows.cap + j0 + row) * a.H + h);
  float *out = (whole ? (float *)a.out : a.part_o) + at * DH;
  const float inv = !whole ? 1.0f : none ? 0.f : 1.0f / l_run;
#pragma unroll
  for (int i = 0; i < OC; ++i) *reinterpret_cast<floatx4 *>(out + 64 * i + 4 * sub) = o[i] * inv;
  if (!whole && sub == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = float2{none && split == 0 ? 0.f : m_run, none && split == 0 ? 1.f : l_run};
}

}  // namespace

// Query tile (32, 64 or 128 packed rows) and key splits.
void attention_quant_plan(DType t, size_t part_elems, AttnArgs *a) {
  const int grp = a->H / a->Hkv;
  const long rows = a->offsets ? ((long)a->rows.cap + a->B - 1) / a->B : a->L, packed = rows * grp;
  a->bq = t == F32 ? 16 : packed <= 32 ? 32 : packed <= 64 ? 64 : 128;
  const int BK = t == F32 ? 32 : 128;
  const long tiles = t == F32 ? ((rows + 15) / 16) * a->B * a->H : ((packed + a->bq - 1) / a->bq) * a->B * a->Hkv;
  long s = (512 + tiles - 1) / (tiles < 1 ? 1 : tiles);
  const long by_keys = ((long)a->L + BK - 1) / BK;
  if (s > by_keys) s = by_keys;
  if (s > 128) s = 128;
  const size_t per_split = (size_t)a->rows.cap * a->H * a->dh;
  if (per_split > 0 && (size_t)s * per_split > part_elems) s = (long)(part_elems / per_split);
  if (s < 1) s = 1;
  a->chunk = split_chunk(a->L, (int)s, BK);
  a->splits = (a->L + a->chunk - 1) / a->chunk;  // drops splits that would be empty
}

void launch_attention_quant(DType t, const AttnArgs &a, const QuantAttn &q, hipStream_t s) {
  if (a.rows.cap <= 0) return;
  if (t == F32) {
    const dim3 grid(max_q_tiles(a, 16), a.H, a.splits);
    if (a.dh == 64 && q.format == Q_E4M3) k_attn_quant_f32<64, Q_E4M3><<<grid, 256, 0, s>>>(a, q);
    else if (a.dh == 64) k_attn_quant_f32<64, Q_INT8><<<grid, 256, 0, s>>>(a, q);
    else if (q.format == Q_E4M3) k_attn_quant_f32<128, Q_E4M3><<<grid, 256, 0, s>>>(a, q);
    else k_attn_quant_f32<128, Q_INT8><<<grid, 256, 0, s>>>(a, q);
  } else if (a.dh == 64) {
    if (a.bq == 32) launch_tile<64, 1, 4>(a, q, s);
    else if (a.bq == 64) launch_tile<64, 2, 2>(a, q, s);
    else launch_tile<64, 4, 1>(a, q, s);
  } else {
    if (a.bq == 32) launch_tile<128, 1, 4>(a, q, s);
    else if (a.bq == 64) launch_tile<128, 2, 2>(a, q, s);
    else launch_tile<128, 4, 1>(a, q, s);
  }
  if (a.splits > 1) launch_attn_combine(t, a, s);
}

}  // namespace dy
