// Kernels on the heads of a row: RMSNorm of query and key heads, rotary embedding and merge into the caches in one pass, the same into
// a cache of 8-bit codes, and that cache read back.  [Alg. 3: q_proj / k_proj / v_proj lines and the K/V merge of layers whose
// queries and keys are normalised]
//
// A head vector x of dh elements:  n = x / sqrt(mean(x^2) + eps) * g;  with the halves n1, n2 and the table's cos, sin of the token's
// position  y1 = n1 cos - n2 sin,  y2 = n2 cos + n1 sin;  sums and products in fp32, one rounding to the storage type or to codes.
// dh / 16 lanes take a vector, a lane 8 neighbouring elements of each half: a pair to be rotated lies in one lane, and the sum of
// squares and the largest magnitude are two or three moves between neighbouring lanes.  A wave takes 64 / (dh / 16) vectors of
// one row.
//
// Bound by memory, every element read and written once: 20480 rows of 12288 columns, bf16 to bf16, 180 us (5.6 TB/s of elements; a copy
// of 4 GiB reaches 4.8); to 8-bit codes, 20480 rows of 8192 columns, 105 us, and back 100 us.  A few hundred rows are bound by the launch:
// 1137 rows of 4608 columns 7.1 us.
#include <type_traits>
#include "common.h"
#include "kernels.h"
#include "quant.h"

namespace dy {

namespace {

constexpr int HB = 256, WPB = HB / WAVE;

template <typename T> __device__ __forceinline__ void load8(const T *p, float *x) {
  constexpr int N = Vec16<T>::N;
#pragma unroll
  for (int i = 0; i < 8 / N; ++i) {
    const Vec16<T> v = ld16(p + i * N);
#pragma unroll
    for (int e = 0; e < N; ++e) x[i * N + e] = v.get(e);
  }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float *x) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4 *>(p) = uint4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  } else {
    *reinterpret_cast<float4 *>(p) = float4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<float4 *>(p + 4) = float4{x[4], x[5], x[6], x[7]};
  }
}

// the largest over the N lanes of a vector, in all of them
template <int N> __device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  x = max(x, moved<0xB1>(x));
  x = max(x, moved<0x4E>(x));
  if (N == 8) x = max(x, moved<0x141>(x));
  return x;
}

// where keys and values go
enum HeadsTo { TO_CACHE = 0, TO_E4M3 = 1, TO_INT8 = 2 };

template <typename T, bool SUMS, int DH, int TO>
__global__ __launch_bounds__(HB) void k_heads(HeadsArgs a) {
  using S = std::conditional_t<SUMS, float, T>;
  constexpr int LPH = DH / 16, HPW = WAVE / LPH, HALF = DH / 2;
  int n = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap;
  Splits sp = a.splits;
  if (SUMS && sp.dev) { sp.n = a.splits.dev[0]; sp.tail_from = a.splits.dev[1]; sp.n_tail = a.splits.dev[2]; }
  const int lane = threadIdx.x % WAVE, sub = lane % LPH;
  const int HT = a.H + 2 * a.Hkv, groups = (HT + HPW - 1) / HPW;
  // a wave to a row's vectors of one group; neighbouring waves take neighbouring groups
  const uint32_t items = (uint32_t)n * (uint32_t)groups;
  for (uint32_t it = blockIdx.x * WPB + threadIdx.x / WAVE; it < items; it += gridDim.x * WPB) {
    const int j = (int)(it / (uint32_t)groups), head = (int)(it % (uint32_t)groups) * HPW + lane / LPH;
    if (head >= HT) continue;  // (whole groups of lanes)
    const int r = a.rows.idx ? a.rows.idx[j] : j;
    const int pos = r % a.L, seq = r / a.L;
    const int kind = head < a.H ? 0 : head < a.H + a.Hkv ? 1 : 2;  // q, k, v
    const int h = kind == 0 ? head : kind == 1 ? head - a.H : head - a.H - a.Hkv;
    const S *src = (const S *)(kind == 0 ? a.q : kind == 1 ? a.k : a.v) + (size_t)j * a.ld + (size_t)h * DH + 8 * sub;
    float x1[8], x2[8];
    load8(src, x1);
    load8(src + HALF, x2);
    if constexpr (SUMS) {
      const size_t stride = (size_t)n * a.ld;
      for (int z = 1; z < sp.of(j); ++z) {
        float y1[8], y2[8];
        load8(src + z * stride, y1);
        load8(src + z * stride + HALF, y2);
#pragma unroll
        for (int e = 0; e < 8; ++e) { x1[e] += y1[e]; x2[e] += y2[e]; }
      }
      const T *b = (const T *)(kind == 0 ? a.bq : kind == 1 ? a.bk : a.bv);
      if (b) {
        float b1[8], b2[8];
        load8(b + (size_t)h * DH + 8 * sub, b1);
        load8(b + (size_t)h * DH + 8 * sub + HALF, b2);
#pragma unroll
        for (int e = 0; e < 8; ++e) { x1[e] += b1[e]; x2[e] += b2[e]; }
      }
    }
    if (kind < 2) {
      const T *g = (const T *)(kind == 0 ? a.g_q : a.g_k);
      if (g) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x2[e], x2[e], fmaf(x1[e], x1[e], ss));
        const float by = 1.0f / sqrtf(lanes_sum<LPH>(ss) * (1.0f / DH) + a.eps);
        float g1[8], g2[8];
        load8(g + 8 * sub, g1);
        load8(g + 8 * sub + HALF, g2);
#pragma unroll
        for (int e = 0; e < 8; ++e) { x1[e] *= by * g1[e]; x2[e] *= by * g2[e]; }
      }
      if (a.tab) {
        const float4 *t = reinterpret_cast<const float4 *>(a.tab + (size_t)pos * DH + 16 * sub);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 cs = t[i];  // cos, sin of two pairs
          const float co[2] = {cs.x, cs.z}, si[2] = {cs.y, cs.w};
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float p = x1[2 * i + u], q = x2[2 * i + u];
            x1[2 * i + u] = rotated(p, co[u], -(q * si[u]));
            x2[2 * i + u] = rotated(q, co[u], p * si[u]);
          }
        }
      }
    }
    if (kind == 0 || TO == TO_CACHE) {
      T *dst = kind == 0 ? (T *)a.q_out + ((size_t)j * a.H + h) * DH
                         : (T *)(kind == 1 ? a.kc : a.vc) + ((size_t)r * a.Hkv + h) * DH;
      store8(dst + 8 * sub, x1);
      store8(dst + 8 * sub + HALF, x2);
    } else if constexpr (TO != TO_CACHE) {
      constexpr int F = TO == TO_E4M3 ? Q_E4M3 : Q_INT8;
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, max(__float_as_uint(x1[e]) & 0x7fffffffu, __float_as_uint(x2[e]) & 0x7fffffffu));
      const QScale qs = q_scale<F>(lanes_max<LPH>(m));
      uint8_t *dst = (kind == 1 ? a.quant.k : a.quant.v) + ((size_t)r * a.Hkv + h) * DH + 8 * sub;
      *reinterpret_cast<uint2 *>(dst) = uint2{q_codes<F>(x1, qs), q_codes<F>(x1 + 4, qs)};
      *reinterpret_cast<uint2 *>(dst + HALF) = uint2{q_codes<F>(x2, qs), q_codes<F>(x2 + 4, qs)};
      if (sub == 0) (kind == 1 ? a.quant.ks : a.quant.vs)[((size_t)seq * a.Hkv + h) * a.L + pos] = qs.scale;
    }
  }
}

// a lane takes 8 neighbouring codes, dh / 8 lanes a vector
template <typename T, int F, int DH>
__global__ __launch_bounds__(HB) void k_quant_read(QuantCache c, Rows rows, int L, int Hkv, T *k_out, T *v_out) {
  constexpr int LPH = DH / 8, HPW = WAVE / LPH;
  const int n = rows.count ? min(*rows.count, rows.cap) : rows.cap;
  const int lane = threadIdx.x % WAVE, sub = lane % LPH;
  const int groups = (2 * Hkv + HPW - 1) / HPW;
  const uint32_t items = (uint32_t)n * (uint32_t)groups;
  for (uint32_t it = blockIdx.x * WPB + threadIdx.x / WAVE; it < items; it += gridDim.x * WPB) {
    const int j = (int)(it / (uint32_t)groups), vec = (int)(it % (uint32_t)groups) * HPW + lane / LPH;
    if (vec >= 2 * Hkv) continue;
    const bool isv = vec >= Hkv;
    const int h = isv ? vec - Hkv : vec;
    const int r = rows.idx ? rows.idx[j] : j;
    const uint2 w = *reinterpret_cast<const uint2 *>((isv ? c.v : c.k) + ((size_t)r * Hkv + h) * DH + 8 * sub);
    const float scale = (isv ? c.vs : c.ks)[((size_t)(r / L) * Hkv + h) * L + r % L];
    float x[8];
    q_values<F>(w.x, scale, x);
    q_values<F>(w.y, scale, x + 4);
    store8((isv ? v_out : k_out) + ((size_t)j * Hkv + h) * DH + 8 * sub, x);
  }
}

// A list's capacity may be far above its count, which the device knows, and workgroups without a row are not free; with fewer of them the
// others take their rows in turn, which costs more: 20480 listed rows of 12288 columns, 2048 / 4096 / 8192 / 16384 / 65536 workgroups
// 207 / 191 / 187 / 179 / 174 us.
inline int grid_of(uint64_t blocks, const Rows &rows) {
  const uint64_t most = rows.count ? 16384 : 1 << 20;
  return (int)(blocks < 1 ? 1 : blocks > most ? most : blocks);
}

}  // namespace

void launch_heads(DType t, const HeadsArgs &a, bool sums, int dh, int to, hipStream_t s) {
  if (a.rows.cap <= 0) return;
  const int hpw = WAVE / (dh / 16), groups = (a.H + 2 * a.Hkv + hpw - 1) / hpw;
  const int grid = grid_of(((uint64_t)a.rows.cap * groups + WPB - 1) / WPB, a.rows);
  auto go = [&](auto zero, auto sums_c, auto dh_c) {
    using T = decltype(zero);
    constexpr bool S = decltype(sums_c)::value;
    constexpr int D = decltype(dh_c)::value;
    if (to == TO_CACHE) k_heads<T, S, D, TO_CACHE><<<grid, HB, 0, s>>>(a);
    else if (to == TO_E4M3) k_heads<T, S, D, TO_E4M3><<<grid, HB, 0, s>>>(a);
    else k_heads<T, S, D, TO_INT8><<<grid, HB, 0, s>>>(a);
  };
  auto by_dh = [&](auto zero, auto sums_c) {
    if (dh == 64) go(zero, sums_c, std::integral_constant<int, 64>{});
    else go(zero, sums_c, std::integral_constant<int, 128>{});
  };
  auto by_sums = [&](auto zero) {
    if (sums) by_dh(zero, std::true_type{});
    else by_dh(zero, std::false_type{});
  };
  if (t == F32) by_sums(float{});
  else by_sums(bf16_t{});
}

void launch_quant_read(DType t, const QuantCache &c, int format, Rows rows, int L, int Hkv, int dh, void *k_out, void *v_out, hipStream_t s) {
  if (rows.cap <= 0) return;
  const int hpw = WAVE / (dh / 8), groups = (2 * Hkv + hpw - 1) / hpw;
  const int grid = grid_of(((uint64_t)rows.cap * groups + WPB - 1) / WPB, rows);
  auto with = [&](auto zero, auto dh_c) {
    using T = decltype(zero);
    constexpr int D = decltype(dh_c)::value;
    if (format == Q_E4M3) k_quant_read<T, Q_E4M3, D><<<grid, HB, 0, s>>>(c, rows, L, Hkv, (T *)k_out, (T *)v_out);
    else k_quant_read<T, Q_INT8, D><<<grid, HB, 0, s>>>(c, rows, L, Hkv, (T *)k_out, (T *)v_out);
  };
  auto go = [&](auto zero) {
    if (dh == 64) with(zero, std::integral_constant<int, 64>{});
    else with(zero, std::integral_constant<int, 128>{});
  };
  if (t == F32) go(float{});
  else go(bf16_t{});
}

}  // namespace dy
