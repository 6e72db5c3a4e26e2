// Requests over pages of keys and values: the page accounting of a step, and the pass over raw projections that writes keys and values into the
// rows' slots.
#include <algorithm>
#include <type_traits>
#include "attention_common.h"
#include "common.h"
#include "kernels.h"

namespace dy {

namespace {

// ---- page accounting ------------------------------------------------------------------------------------
// held = ceil(len / P), need = ceil(new_len / P); loss = held - need and gain = need - held where positive.  Three prefix sums over the
// requests (rows, gains, losses) say everything: released page k is entry need + k - (losses before) of the request it falls into, taken
// page k is released page k while there are any and then comes from the top of the free list, and a row's slot needs the one page its
// position lies in.  So the sums are made once a workgroup, in LDS, and rows, taken pages and pages that go back to the list are dealt out
// by their numbers, each finding its request by a binary search: no workgroup waits for another, long prompts are shared out, and the
// result does not depend on the order of anything.
// Bound by the launch and the chain load - scan - search - load - store: 64 decoded tokens 2.7 us, 1500 requests with chunks of up to 512 tokens 9.4
// (medians of a kernel trace).
constexpr int MANY = 1 << 30;  // sums stop here
__device__ __forceinline__ int sat(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)MANY); }
template <int CTRL, int ROWS> __device__ __forceinline__ int sat_step(int x) {
  return sat(x, __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int sat_scan(int x) {  // inclusive over a wave, as wave_scan
  x = sat_step<0x111, 0xf>(x);
  x = sat_step<0x112, 0xf>(x);
  x = sat_step<0x114, 0xf>(x);
  x = sat_step<0x118, 0xf>(x);
  x = sat_step<0x142, 0xa>(x);
  return sat_step<0x143, 0xc>(x);
}
// first r with v[r] > k, v ascending; n if none
__device__ __forceinline__ int first_above(const int *v, int n, int k) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if (v[m] > k) hi = m; else lo = m + 1;
  }
  return lo;
}

// MOST requests; up to 2048 all that later steps ask of a request lies in LDS, beyond that the sums alone
template <int NT, int MOST>
__global__ __launch_bounds__(NT) void k_page_plan(Pages pages, PagePlan a) {
  constexpr bool KEPT = MOST <= 2048;
  constexpr int NW = NT / WAVE;
  __shared__ int rows_to[MOST], gain_to[MOST], loss_to[MOST];  // inclusive sums
  __shared__ int kept[KEPT ? 3 * MOST : 1];                    // first position of a row (-1 - that: without room), held, need
  __shared__ int wave_total[3][NW];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), R = a.R;
  const int shift = pages.shift, room = pages.max_pages << shift;  // (at most 2^30: checked on the host)
  const int free_word = a.n_free[0];
  struct Req { int start, held, need; bool fits; };  // start: position of its first row
  struct Full { Req q; int rows, len, then; };
  auto read = [&](int r) {
    Full f;
    f.len = min(max(a.len[r], 0), room);
    const int want = max(a.new_len[r], 0);
    f.q.fits = want <= room;
    f.then = f.q.fits ? want : f.len;
    f.rows = min(max(a.new_rows[r], 0), f.then);
    f.q.start = f.then - f.rows;
    f.q.held = (f.len + (1 << shift) - 1) >> shift;
    f.q.need = (f.then + (1 << shift) - 1) >> shift;
    return f;
  };
  auto request = [&](int r) {
    if constexpr (KEPT) {
      const int s = kept[r];
      return Req{s < 0 ? -1 - s : s, kept[MOST + r], kept[2 * MOST + r], s >= 0};
    } else {
      return read(r).q;
    }
  };
  int carry[3] = {0, 0, 0};
  bool unfit = false;
  for (int r0 = 0; r0 < R; r0 += NT) {
    const int r = r0 + tid;
    int x[3] = {0, 0, 0};
    if (r < R) {
      const Full f = read(r);
      x[0] = f.rows;
      x[1] = max(f.q.need - f.q.held, 0);
      x[2] = max(f.q.held - f.q.need, 0);
      unfit = unfit || !f.q.fits;
      if constexpr (KEPT) {
        kept[r] = f.q.fits ? f.q.start : -1 - f.q.start;
        kept[MOST + r] = f.q.held;
        kept[2 * MOST + r] = f.q.need;
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) x[i] = sat_scan(x[i]);
    if (r0) __syncthreads();
    if (lane == WAVE - 1)
#pragma unroll
      for (int i = 0; i < 3; ++i) wave_total[i][wave] = x[i];
    __syncthreads();
    int *to[3] = {rows_to, gain_to, loss_to};
#pragma unroll
    for (int i = 0; i < 3; ++i) {  // (the totals of the waves, summed up by each of them)
      const int upto = sat_scan(lane < NW ? wave_total[i][lane] : 0);
      const int before = wave ? __builtin_amdgcn_readlane(upto, wave - 1) : 0;
      if (r < R) to[i][r] = sat(sat(carry[i], before), x[i]);
      carry[i] = sat(carry[i], __builtin_amdgcn_readlane(upto, NW - 1));
    }
  }
  __syncthreads();
  // (below MANY, so that a sum of gains that has stopped there is more than there are)
  const int released = carry[2], n_free = min(max(free_word, 0), pages.n_pages), have = min(sat(n_free, released), MANY - 1);
  // pages taken: the gains of the served requests, which are a prefix of those that gain
  int taken = carry[1];
  if (taken > have) {
    const int r = first_above(gain_to, R, have);
    taken = r ? gain_to[r - 1] : 0;
  }
  const int n_rows = min(carry[0], a.cap), left = max(released - taken, 0);
  if (unfit || (tid == 0 && blockIdx.x == 0 && (carry[1] > have || carry[0] > a.cap))) *a.status = a.overflow_code;

  auto before_of = [](const int *v, int r) { return r ? v[r - 1] : 0; };
  auto released_page = [&](int k) {
    const int r = first_above(loss_to, R, k);
    return pages.table[(size_t)r * pages.max_pages + request(r).need + (k - before_of(loss_to, r))];
  };
  auto taken_page = [&](int k) { return k < released ? released_page(k) : a.free_list[n_free - 1 - (k - released)]; };
  auto served = [&](int r, const Req &q) { return q.fits && (q.need <= q.held || gain_to[r] <= have); };  // (two sums say nothing where both have stopped)
  // rows, table entries gained, pages that go back, requests: one after the other in number (each at most MANY: 32 bits hold their sum)
  const uint32_t total = (uint32_t)n_rows + (uint32_t)taken + (uint32_t)left + (uint32_t)R;
  for (uint32_t i = blockIdx.x * NT + tid; i < total; i += gridDim.x * NT) {
    if (i < (uint32_t)n_rows) {
      const int k = (int)i;
      const int r = first_above(rows_to, R, k);
      const Req q = request(r);
      const int p = q.start + (k - before_of(rows_to, r)), e = p >> shift;
      a.pos[k] = p;
      int slot = -1;
      if (served(r, q)) {
        const int page = e < q.held ? pages.table[(size_t)r * pages.max_pages + e] : taken_page(before_of(gain_to, r) + (e - q.held));
        slot = (int)(((uint32_t)page << shift) | (uint32_t)(p & ((1 << shift) - 1)));
      }
      a.slot[k] = slot;
      continue;
    }
    uint32_t rest = i - (uint32_t)n_rows;
    if (rest < (uint32_t)taken) {
      const int k = (int)rest;
      const int r = first_above(gain_to, R, k);
      pages.table[(size_t)r * pages.max_pages + request(r).held + (k - before_of(gain_to, r))] = taken_page(k);
      continue;
    }
    rest -= (uint32_t)taken;
    if (rest < (uint32_t)left) {
      const int k = (int)rest, at = sat(n_free, k);
      if (at < pages.n_pages) a.free_list[at] = released_page(taken + k);
      continue;
    }
    const int k = (int)(rest - (uint32_t)left);
    if (k == 0) {
      a.offsets[0] = 0;
      a.n_free_out[0] = min(have - taken, pages.n_pages);
    }
    const Full f = read(k);
    a.len_out[k] = served(k, f.q) ? f.then : f.len;
    a.offsets[k + 1] = min(rows_to[k], a.cap);
  }
}

// ---- head norms, rotation on several axes, keys and values into slots ---------------------------------------------
// As k_heads (headops.hip) takes a head: dh / 16 lanes, 8 neighbouring columns of each half a lane.  Here a wave takes `per` groups of
// heads of one row, and with them the row's angles once: a lane computes cosine and sine of one pair and leaves them in LDS.
//   angle = pos * f turns, f = theta^(-2p/dh) / 2 pi, held in 2^-64 turns: the product modulo 2^64 is the angle's fraction of a turn with whole
// turns gone, right to 2^-31 turns at any 32-bit position (the factor's rounding times the position, and the low word that
// is cut off: 2^-32 each).  Its nearest quarter turn leaves |x| <= pi / 4, where the series of sine and
// cosine end with x^9 and x^10 (what is left out is below 2e-9 and 2e-10).
// Bound by the rows' way in and out: 8192 rows of 32 + 2 x 32 heads of 128 in bf16, 403 MB, 76 us (5.3 TB/s); of few rows by the launch (3 us).
__device__ __forceinline__ float2 cos_sin(uint64_t f, int pos) {
  const uint32_t t = (uint32_t)((f * (uint64_t)(int64_t)pos) >> 32);
  const uint32_t q = (t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(t - (q << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.0f);
  const float co = q & 1 ? s : c, si = q & 1 ? c : s;
  return float2{(q + 1) & 2 ? -co : co, q & 2 ? -si : si};
}

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

constexpr int PH_NT = 256, PH_WAVES = PH_NT / WAVE;

template <typename T, int DH>
__global__ __launch_bounds__(PH_NT) void k_heads_paged(PagedHeads a, int per, int parts) {
  constexpr int LPH = DH / 16, HPW = WAVE / LPH, HALF = DH / 2;
  __shared__ float2 table[PH_WAVES][HALF];
  const int n = max(min(*a.rows.count, a.rows.cap), 0);
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, sub = lane % LPH;
  const int HT = a.H + 2 * a.Hkv, P = 1 << a.pages.shift;
  const long slots = (long)a.pages.n_pages << a.pages.shift;
  const uint32_t items = (uint32_t)n * (uint32_t)parts;
  for (uint32_t it = blockIdx.x * PH_WAVES + wave; it < items; it += gridDim.x * PH_WAVES) {
    const int j = (int)(it / (uint32_t)parts), g0 = (int)(it % (uint32_t)parts) * per;
    const int slot = a.slot[j];
    if (lane < HALF) table[wave][lane] = cos_sin(a.turns[lane], a.pos[(size_t)a.axis[lane] * a.rows.cap + j]);
    if (slot >= slots && lane == 0) *a.status = a.bad_slot_code;
    const bool keep = slot >= 0 && slot < slots;
    const size_t page = (size_t)((uint32_t)slot >> a.pages.shift), place = (uint32_t)slot & (P - 1);
    __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses keep their order)
    float co[8], si[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 cs = table[wave][8 * sub + e];
      co[e] = cs.x; si[e] = cs.y;
    }
    __builtin_amdgcn_wave_barrier();
    const T *row = (const T *)a.qkv + (size_t)j * a.ld + 8 * sub;
    for (int g = g0; g < g0 + per; ++g) {
      const int head = g * HPW + lane / LPH;
      if (head >= HT) break;  // (whole groups of lanes)
      const int kind = head < a.H ? 0 : head < a.H + a.Hkv ? 1 : 2;  // q, k, v
      float x1[8], x2[8];
      load8(row + (size_t)head * DH, x1);
      load8(row + (size_t)head * DH + HALF, x2);
      if (kind < 2) {
        const T *gain = (const T *)(kind == 0 ? a.g_q : a.g_k);
        if (gain) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(x2[e], x2[e], fmaf(x1[e], x1[e], ss));
          const float by = 1.0f / sqrtf(lanes_sum<LPH>(ss) * (1.0f / DH) + a.eps);
          float g1[8], g2[8];
          load8(gain + 8 * sub, g1);
          load8(gain + 8 * sub + HALF, g2);
#pragma unroll
          for (int e = 0; e < 8; ++e) { x1[e] *= by * g1[e]; x2[e] *= by * g2[e]; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = x1[e], q = x2[e];
          x1[e] = rotated(p, co[e], -(q * si[e]));
          x2[e] = rotated(q, co[e], p * si[e]);
        }
      }
      T *dst;
      if (kind == 0) {
        dst = (T *)a.q_out + ((size_t)j * a.H + head) * DH;
      } else {
        if (!keep) continue;
        const int h = head - a.H - (kind == 2 ? a.Hkv : 0);
        dst = (T *)(kind == 1 ? a.pages.k : a.pages.v) + ((page * a.Hkv + h) * P + place) * DH;
      }
      store8(dst + 8 * sub, x1);
      store8(dst + 8 * sub + HALF, x2);
    }
  }
}

}  // namespace

// Rows are shared out over workgroups that each make the sums, so more of them than rows keep busy only add sums.
void launch_page_plan(const Pages &pages, const PagePlan &a, hipStream_t s) {
  const long work = (long)a.cap + a.R;
  const bool small = a.R <= 256;
  const int nt = small ? 256 : 1024;
  const long blocks = (work + 2 * nt - 1) / (2 * nt);
  const int grid = (int)(blocks < 1 ? 1 : blocks > 256 ? 256 : blocks);
  if (small) k_page_plan<256, 256><<<grid, 256, 0, s>>>(pages, a);
  else if (a.R <= 2048) k_page_plan<1024, 2048><<<grid, 1024, 0, s>>>(pages, a);
  else k_page_plan<1024, MAX_REQUESTS><<<grid, 1024, 0, s>>>(pages, a);
}

void launch_heads_paged(DType t, const PagedHeads &a, int dh, hipStream_t s) {
  if (a.rows.cap <= 0) return;
  const int hpw = WAVE / (dh / 16), groups = (a.H + 2 * a.Hkv + hpw - 1) / hpw;
  // Groups of a wave, which share a row's angles.  1 / 2 / 4 / all of them, us, heads of 128: 64 rows of 96 heads 3.2 / 3.8 / 5.0 / 9.2; 512 rows
  // 7.4 / 7.3 / 8.4 / 13; 1277 of 36 heads 8.4 / 7.7 / 7.7 / 8.5; 8192 of 96 77 / 75 / 78 / 86.
  long per = (long)a.rows.cap * groups >= 4096 ? std::min(2, groups) : 1;
  const int parts = (int)((groups + per - 1) / per);
  per = (groups + parts - 1) / parts;
  const uint64_t blocks = ((uint64_t)a.rows.cap * parts + PH_WAVES - 1) / PH_WAVES;
  const int grid = (int)(blocks > (1 << 20) ? 1 << 20 : blocks);
  auto go = [&](auto zero) {
    using T = decltype(zero);
    if (dh == 64) k_heads_paged<T, 64><<<grid, PH_NT, 0, s>>>(a, (int)per, parts);
    else k_heads_paged<T, 128><<<grid, PH_NT, 0, s>>>(a, (int)per, parts);
  };
  if (t == F32) go(float{});
  else go(bf16_t{});
}

}  // namespace dy
