// The 8-bit key/value cache: per (token, key-value head) a vector of dh codes and one fp32 scale; value = code * scale.
//   e4m3  the scale is a power of two, 2^max(e, -100) with the smallest e for which max|x| / 2^e <= 448.  Nothing is lost by that (the
//         codes are floating point: a larger scale costs their smallest subnormals alone), every quotient is exact before its one
//         rounding, a value read back and written again has the same code, code * scale is exact in bf16, and the conversion
//         to bf16 takes the scale along in one instruction.
//   int8  m = max(max|x|, 2^-100), scale = m / 127, code = rint(x * (127 / m)).
// A vector with an infinity or NaN has a NaN for its scale and codes 0, so that it reads back as NaN.
#pragma once
#include "common.h"

namespace dy {

enum QFormat { Q_E4M3 = 0, Q_INT8 = 1 };

struct QuantCache {
  uint8_t *k = nullptr, *v = nullptr;     // [B, L, Hkv, dh] codes
  float *ks = nullptr, *vs = nullptr;     // [B, Hkv, L] scales
};

// Scale of a vector and what its elements are multiplied by, from the bits of its largest magnitude.  (As integers the bits of magnitudes
// order as the magnitudes do, infinities and NaN above all others.)
struct QScale { float scale, inv; };
template <int F> __device__ __forceinline__ QScale q_scale(uint32_t m) {
  if (m >= 0x7f800000u) return QScale{__uint_as_float(0x7fc00000u), 0.f};
  m = max(m, (127u - 100u) << 23);
  if constexpr (F == Q_E4M3) {  // 448 = 1.75 * 2^8
    const int e = max((int)(m >> 23) - 127 - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
    return QScale{__uint_as_float((uint32_t)(127 + e) << 23), __uint_as_float((uint32_t)(127 - e) << 23)};
  } else {
    const float f = __uint_as_float(m);
    return QScale{f / 127.0f, 127.0f / f};
  }
}

// four elements -> four codes, nearest even  (q.inv is 0 only where an element may be no number: codes 0)
template <int F> __device__ __forceinline__ uint32_t q_codes(const float *x, const QScale &q) {
  if (q.inv == 0.f) return 0u;
  if constexpr (F == Q_E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * q.inv, x[1] * q.inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * q.inv, x[3] * q.inv, w, true);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)rintf(x[i] * q.inv) & 0xffu) << (8 * i);
    return w;
  }
}

// four codes -> four values
template <int F> __device__ __forceinline__ void q_values(uint32_t w, float scale, float *x) {
  if constexpr (F == Q_E4M3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0] * scale; x[1] = lo[1] * scale; x[2] = hi[0] * scale; x[3] = hi[1] * scale;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i)) * scale;
  }
}

// four codes -> four bf16 values in two words, exact.  e4m3: the values, of the scale the exponent alone (a NaN gives NaN).  int8: the
// codes, whose scales are applied to what is made of them.
template <int F> __device__ __forceinline__ uint2 q_bf16(uint32_t w, float scale) {
  if constexpr (F == Q_E4M3) {
    return uint2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
  } else {
    return uint2{pack_bf16((float)(int8_t)w, (float)(int8_t)(w >> 8)), pack_bf16((float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24))};
  }
}

}  // namespace dy
