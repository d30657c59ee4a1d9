// From the logits to the next tokens: penalties, bias and allowed tokens, and the draw.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>

#include "tmz_device.h"
#include "tmz_internal.h"

namespace tmz {

constexpr int32_t kErrRules = 64, kErrSample = 128;      // bits of the deferred error word

template <int N>
struct __attribute__((packed, aligned(4))) Floats {      // rows of any length begin at any multiple of 4 bytes
  float v[N];
};
typedef Floats<4> Four;
struct __attribute__((packed, aligned(4))) Ids {
  int32_t v[4];
};

// ---------------------------------------------------------------------------
// Rules on the logits, a work group for a slice of a row.  The history's tokens that fall into the slice
// are counted in LDS (bit 0: a prompt token, the rest: how often generated), so that no counter of the
// vocabulary's size passes through memory and the counts do not depend on the order.  Then every logit is
// read, adjusted and written once: bound by these bytes.
// ---------------------------------------------------------------------------
struct RuleArgs {
  const float* logits;
  float* out;
  int32_t vocab;
  termezo_logit_rules r;
  int32_t* err;
};

// Line of a table that row takes: -1 none.
__device__ __forceinline__ int rule_line(const int32_t* index, int lines, int row, bool& bad) {
  const int i = index ? index[row] : (lines == 1 ? 0 : row);
  if (i >= -1 && i < lines) return i;
  bad = true;
  return -1;
}

// A slice of a row, 4 * E values of a thread: raw[i].v[j] at t0 + PASS i + 4 tid + j; `none` behind the row's end.
template <int E, int PASS = 1024>
__device__ __forceinline__ void slice_fetch(const float* row, int t0, int V, int tid, float none, Four raw[E]) {
  const uint32_t at = (uint32_t)t0 + 4u * tid;
  if (t0 + PASS * E <= V) {                              // whole work group
#pragma unroll
    for (int i = 0; i < E; ++i) raw[i] = *(const Four*)(row + (at + (uint32_t)PASS * i));
    return;
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint32_t t = at + (uint32_t)PASS * i;
    raw[i] = Four{{none, none, none, none}};
    if (t + 4u <= (uint32_t)V) {
      raw[i] = *(const Four*)(row + t);
    } else if (t < (uint32_t)V) {
      raw[i].v[0] = row[t];
      if (t + 1u < (uint32_t)V) raw[i].v[1] = row[t + 1u];
      if (t + 2u < (uint32_t)V) raw[i].v[2] = row[t + 2u];
    }
  }
}

// SLICE logits a work group: 1024 where that gives a compute unit four work groups at most (latency counts); else 8192
// with a history, which every slice of a row goes through (64 x 128256, 4000 tokens: 16.6 us, 18.5 with 4096, 23.5 with
// 16384), 4096 without (192 x 32000 with bias and mask: 9.8 us, 5.1 TB/s; 10.9 with 8192).  With the logits on
// their way while the history is counted the registers leave too few waves: 16.6 -> 19 us.
template <int SLICE, bool HIST>
__global__ void __launch_bounds__(256) k_adjust(RuleArgs a) {
  __shared__ uint32_t count[HIST ? SLICE : 1];
  const int tid = threadIdx.x, row = blockIdx.y, V = a.vocab;
  const int t0 = blockIdx.x * SLICE, n = min(SLICE, V - t0);
  bool bad = false;
  int64_t len = a.r.hist_len, from = 0;
  if (HIST && a.r.lengths) len = a.r.lengths[row];
  if (HIST && a.r.starts) from = a.r.starts[row];
  const float rep = HIST && a.r.repetition ? a.r.repetition[row] : 1.0f;
  const float freq = HIST && a.r.frequency ? a.r.frequency[row] : 0.0f;
  const float pres = HIST && a.r.presence ? a.r.presence[row] : 0.0f;
  const int bl = a.r.bias ? rule_line(a.r.bias_index, a.r.n_bias, row, bad) : -1;
  const int ml = a.r.mask ? rule_line(a.r.mask_index, a.r.n_masks, row, bad) : -1;
  if (HIST)
    for (int i = tid; i < n; i += 256) count[i] = 0u;
  if (HIST) {
    if (len < 0 || len > a.r.hist_len || from < 0 || from > len) {
      bad = true;
      len = 0;
    }
    __syncthreads();
    const int32_t* h = a.r.history + row * a.r.hist_len;
    auto one = [&](int32_t id, int64_t i) __attribute__((always_inline)) {
      const uint32_t at = (uint32_t)id - (uint32_t)t0;   // ids outside the vocabulary are outside every slice
      if (at < (uint32_t)n) {
        if (i >= from) atomicAdd(&count[at], 2u);
        else atomicOr(&count[at], 1u);
      }
    };
    for (int64_t i0 = 4 * tid; i0 < len; i0 += 4096) {
      Ids id[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t i = i0 + 1024 * k;
        if (i + 4 <= len) {
          id[k] = *(const Ids*)(h + i);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) id[k].v[j] = i + j < len ? h[i + j] : -1;
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) one(id[k].v[j], i0 + 1024 * k + j);
    }
    __syncthreads();
  }
  if (bad && tid == 0 && blockIdx.x == 0) atomicOr(a.err, kErrRules);
  const float* x = a.logits + (int64_t)row * V;
  float* y = a.out + (int64_t)row * V;
  const float* bias = bl >= 0 ? a.r.bias + (int64_t)bl * V : nullptr;
  const uint32_t* mask = ml >= 0 ? a.r.mask + (int64_t)ml * ((V + 31) / 32) : nullptr;
  auto one = [&](float v, int i, float b, uint32_t allowed) __attribute__((always_inline)) {
    if (HIST) {
      const uint32_t c = count[i];
      if (c) {
        v = v > 0.0f ? __fdiv_rn(v, rep) : v * rep;
        if (c > 1u) {
          v = v - (float)(c >> 1) * freq;
          v = v - pres;
        }
      }
    }
    if (bias) v = v + b;
    return allowed & 1u ? v : -INFINITY;
  };
  for (int i = tid * 4; i < n; i += 1024) {
    const int t = t0 + i;
    const uint32_t bits = mask ? mask[t >> 5] >> (t & 31) : 15u;
    if (i + 3 < n) {
      Four f = *(const Four*)(x + t), b = {};
      if (bias) b = *(const Four*)(bias + t);
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = one(f.v[j], i + j, b.v[j], bits >> j);
      *(Four*)(y + t) = f;
    } else {
      for (int j = 0; i + j < n; ++j) y[t + j] = one(x[t + j], i + j, bias ? bias[t + j] : 0.0f, bits >> j);
    }
  }
}

// ---------------------------------------------------------------------------
// The draw.  Every limit keeps a beginning of the row's order (falling logits, equal ones by index), so
// what is kept is one border in that order; the token then comes from the prefix sums of the kept weights in
// the order of indices.
//
// k_draw_scan, a work group for a slice of a row: the slice's largest logit m_s, its weights exp((x - m_s) / T),
// their sum, and sums and counts by bins (in fixed point: integer sums do not depend on their order).
// A bin is an eighth of T wide on a grid that all slices share (bin = floor(x (8 / T))), counted from the slice's
// best bin downwards; the last of the 256 holds all that lies lower.
// k_draw_list, the same grid: the row's bins (slices weighted by exp((m_s - m) / T)) tell in which of them the
// borders lie (long slices: found by k_draw_plan before); the slice's logits in those bins go to the row's list.
// k_draw_pick, a work group a row: finds the border in the list by narrowing a range of keys (logit, index),
// a part a thread at a time; then the slice and the token.  Where the list does not hold them it goes through the
// row in the list's place, alone: many equal logits; a top_k whose border lies 32 T and more below the best logit, all of which is
// the last bin (a confident row, a low temperature); bins with many tokens (flat rows of a large vocabulary).  64 x 128256 of
// deviation 2.5 with one logit at 24, T = 0.3, top_k up to 100: 500 us, 40 without that logit; one such row 630 (26); one row of
// 262144 of deviation 1 with top_p 1270 us, of deviation 2.5 41.
// Without limits the first and the last are enough.
// The scan is bound by vector instructions (an exponential in fp64 and a bin a logit) beside its reads, the list by
// its reads, the plan and the pick by their chains of barriers: 64 x 128256 with top_p 14.3 + 5.9 + 12.3 + 20.4 us (the logits
// alone at the rate of a copy: 6.4), one row of 32003 with top_k and top_p 3.8 + 8.2 + 9.4, 256 x 32000 without
// limits 11.3 + 5.2.
// ---------------------------------------------------------------------------
constexpr int kBins = 256, kMaxDrawRows = 1024, kList = 8192;
constexpr bool plan_first(int E) { return E > 2; }       // long slices: plans in a launch of their own
constexpr int kCopies = 4;           // of the bins, so that neighbouring lanes seldom meet in one
// A slice's sums by bins are formed in units of 2^-51 of its largest weight (a copy holds those of 2048 logits) and
// kept in units of 2^-50: 8192 weights are off by 8192 * 2^-52 and a bin by 2^-51, together less than 2^-38.9 of that weight.
constexpr double kScanUnit = 0x1p51, kSliceUnit = 0x1p50;
constexpr double kLog2e32 = 32.0 * 0x1.71547652b82fep+0, kLn2by32 = 0x1.62e42fefa39efp-6;   // 32 log2(e), ln(2) / 32

struct SliceStat {
  float top;                         // -inf: nothing
  int32_t bin;
  double sum;                        // weights relative to top
};
struct RowPlan {                     // what k_draw_list found
  float top, xm;                     // the row's largest logit; the least one that min_p keeps
  // the least logit of the bins before first, of those up to last, before limit, up to limit (NaN: there is none)
  float x_first, x_last, x_before, x_limit;
  int32_t bin;
  // Bins before first are kept; listed are bins first .. last, where top_p's border lies (or the only one), and
  // bin limit, where top_k or min_p ends (kBins: they do not)
  int32_t first, last, limit;
  int32_t count1;                    // tokens in the bins before limit
  double mass0, mass1;               // weights (relative to top) in the bins before first, before limit
  double total;                      // of the whole row
};

struct DrawArgs {
  const float *logits, *uniforms, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens;
  float* logprobs;
  int32_t vocab, slices;
  SliceStat* stat;                   // [rows][slices]
  double* sure;                      // [rows][slices]: a slice's weights in the row's bins before first
  unsigned long long* mass;          // [rows][slices][kBins]
  uint32_t* count;
  RowPlan* plan;                     // [rows]
  int32_t* listed;                   // [rows]
  unsigned long long* list;          // [rows][kList]
  int32_t* err;
};

struct Settings {
  double inv_t, scale;               // 1 / T and kLog2e32 / T
  float grid;                        // 8 / T
  float p, min_p;                    // p 1: none; min_p 0: none
  int k;                             // 0: none
  bool best, bad;                    // best: the best token alone
};

__device__ __forceinline__ Settings draw_settings(const DrawArgs& a, int row) {
  Settings s;
  float t = a.temperature ? a.temperature[row] : 1.0f;
  s.k = a.top_k ? max(a.top_k[row], 0) : 0;
  if (s.k >= a.vocab) s.k = 0;
  s.p = a.top_p ? a.top_p[row] : 1.0f;
  s.min_p = a.min_p ? a.min_p[row] : 0.0f;
  s.bad = !(t >= 0.0f && t <= FLT_MAX) || s.p != s.p || s.min_p != s.min_p;
  if (!(s.p < 1.0f)) s.p = 1.0f;
  if (!(s.min_p > 0.0f)) s.min_p = 0.0f;
  s.best = !(t > 0.0f && t <= FLT_MAX);
  if (s.best) {
    t = 1.0f;
    s.k = 1;
    s.p = 1.0f;
    s.min_p = 0.0f;
  }
  if (s.min_p > 1.0f) s.k = 1;                           // no weight reaches it: the first one is kept
  s.inv_t = 1.0 / (double)t;
  s.scale = kLog2e32 * s.inv_t;
  s.grid = fminf(8.0f / t, FLT_MAX);
  return s;
}

// NaN is -inf, +inf the largest number, -0 is 0.
__device__ __forceinline__ float draw_clean(float x) { return fminf(fmaxf(x + 0.0f, -INFINITY), FLT_MAX); }
__device__ __forceinline__ int draw_bin(float x, float grid) {
  return (int)__builtin_amdgcn_fmed3f(floorf(x * grid), -1e9f, 1e9f);
}
// exp(z) for z <= 0, given q = 32 z log2(e): q = n + f, |f| <= 1/2; 2^(n / 32) from a table of 2^(j / 32) whose entries
// lie on LDS banks of their own, 2^(f / 32) from its series: f^5, the last term that counts, is replaced by the polynomial of
// lower degree that is nearest to it on [-1/2, 1/2] (f^5 - T5(2 f) / 512), which leaves less than 2^-43.  fp64
// throughout; half the operations of a series without a table.
constexpr int kRootCount = 32;
__device__ const double kRoots[kRootCount] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};
__device__ __forceinline__ double exp_of(double q, const double* roots) {     // q >= -32000: no denormals
  constexpr double l = kLn2by32, l5 = l * l * l * l * l / 120;
  const double shifted = q + 0x1.8p52;                   // rounded to a whole number n
  const int n = (int)(uint32_t)__double_as_longlong(shifted);
  const double f = q - (shifted - 0x1.8p52);
  double p = l * l * l * l / 24;
  p = fma(p, f, l * l * l / 6 + l5 * 0.3125);
  p = fma(p, f, l * l / 2);
  p = fma(p, f, l - l5 * 0.01953125);
  p = fma(p, f, 1.0);
  const double w = p * roots[n & (kRootCount - 1)];
  return __hiloint2double(__double2hiint(w) + ((n >> 5) << 20), __double2loint(w));
}
// The weight of x beside top: exp((x - top) / T), scale = kLog2e32 / T.  -inf has 0, or what rounds to it.
__device__ __forceinline__ double draw_weight(float x, float top, double scale, const double* roots) {
  return exp_of(fmax(((double)x - (double)top) * scale, -32000.0), roots);
}
// The least logit with a weight: 2^-1000 of the best one's.  A token masked with the type's lowest value weighs nothing, and is
// not the first one up to which the weights exceed 0 (u = 0, once in 2^24 draws).
__device__ __forceinline__ float draw_floor(float top, const Settings& s) {
  return fmaxf(__double2float_ru((double)top - 693.1471805599453 / s.inv_t), -FLT_MAX);           // 1000 ln 2
}
// ln x for x >= 2^-60: x = 2^e m with m from 0.7 to 1.42, ln m = 2 artanh((m - 1) / (m + 1)) by its series up to the 15th
// power of a quotient below 0.18 (what is left out is below 2^-44).  Inline and short: the general function's code
// had to come from memory for its one call.
__device__ __forceinline__ double ln_of(double x) {
  const int hi = __double2hiint(x), e = (hi - 0x3FE6A09E) >> 20;
  const double m = __hiloint2double(hi - (e << 20), __double2loint(x)), t = (m - 1.0) / (m + 1.0), q = t * t;
  double p = 1.0 / 15;
  p = fma(p, q, 1.0 / 13);
  p = fma(p, q, 1.0 / 11);
  p = fma(p, q, 1.0 / 9);
  p = fma(p, q, 1.0 / 7);
  p = fma(p, q, 1.0 / 5);
  p = fma(p, q, 1.0 / 3);
  return fma((double)e, 0x1.62e42fefa39efp-1, 2.0 * fma(t * q, p, t));
}
// w in [0, 1] in units of 2^-51, rounded to nearest.
__device__ __forceinline__ unsigned long long scan_fix(double w) {
  return (unsigned long long)__double_as_longlong(fma(w, kScanUnit, 0x1p52)) & ((1ull << 52) - 1);
}
// A bin's sum over its copies, from units of 2^-51 to units of 2^-50 (up to 2^63).
__device__ __forceinline__ unsigned long long scan_sum(const unsigned long long* copies) {
  unsigned long long m = 0, low = 0;
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const unsigned long long c = copies[i * kBins];
    m += c >> 1;
    low += c & 1;
  }
  return m + (low >> 1);
}
// The unit of the listed weights: a power of two that takes a row's whole weight (1 to 2^24) to 2^62 .. 2^63, so that each of
// them is off by at most 2^-63 of the whole, however small it is beside the largest, and all of them by 2^-39.
__device__ __forceinline__ double list_unit(double total) {
  return __hiloint2double((2 * 1023 + 62 - (__double2hiint(total) >> 20)) << 20, 0);
}
__device__ __forceinline__ unsigned long long list_fix(double w, double unit) { return __double2ull_rn(w * unit); }
// Keys in the order of the row: greater comes first.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ unsigned long long draw_key(float x, int t) {
  return (unsigned long long)ordered(x) << 32 | (0xFFFFFFFFu - (uint32_t)t);
}
__device__ __forceinline__ float key_logit(unsigned long long k) { return unordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_token(unsigned long long k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// v of the lane that a data-parallel move names, `none` where there is no such lane or its row is left out.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T moved(T v, T none) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "32 or 64 bits");
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL,
                                                             ROWS, 0xF, false));
  } else {
    typedef int v2i __attribute__((ext_vector_type(2)));
    const v2i a = __builtin_bit_cast(v2i, v), o = __builtin_bit_cast(v2i, none);
    return __builtin_bit_cast(T, v2i{__builtin_amdgcn_update_dpp(o[0], a[0], CTRL, ROWS, 0xF, false),
                                     __builtin_amdgcn_update_dpp(o[1], a[1], CTRL, ROWS, 0xF, false)});
  }
}
// The lane up to and including which v is combined by f: steps of 1, 2, 4 and 8 within rows of 16 lanes, then each
// row's last lane to the next row, then lane 31 to the upper half (a shuffle through LDS takes ten times as long).
template <typename T, typename F>
__device__ __forceinline__ T wave_fold(T v, T none, F f) {
  v = f(v, moved<0x111, 0xF>(v, none));
  v = f(v, moved<0x112, 0xF>(v, none));
  v = f(v, moved<0x114, 0xF>(v, none));
  v = f(v, moved<0x118, 0xF>(v, none));
  v = f(v, moved<0x142, 0xA>(v, none));
  v = f(v, moved<0x143, 0xC>(v, none));
  return v;
}
template <typename T>
__device__ __forceinline__ T last_lane(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
  } else {
    typedef int v2i __attribute__((ext_vector_type(2)));
    const v2i a = __builtin_bit_cast(v2i, v);
    return __builtin_bit_cast(T, v2i{__builtin_amdgcn_readlane(a[0], 63), __builtin_amdgcn_readlane(a[1], 63)});
  }
}
// Inclusive prefix sums over the wave's lanes, and results of all of them in every lane.
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
  return wave_fold(v, (T)0, [](T a, T b) __attribute__((always_inline)) { return a + b; });
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
  return last_lane(wave_scan(v));
}
__device__ __forceinline__ float wave_top(float v) {
  return last_lane(wave_fold(v, -INFINITY, [](float a, float b) __attribute__((always_inline)) { return fmaxf(a, b); }));
}

// LIMITS: bins are wanted, COUNT: their tokens are counted too (top_k).
template <int E, bool LIMITS, bool COUNT>
__global__ void __launch_bounds__(256) k_draw_scan(DrawArgs a) {
  __shared__ unsigned long long mass[LIMITS ? kCopies * kBins : 1];
  __shared__ double sums[4];
  __shared__ uint32_t count[COUNT ? kCopies * kBins : 1];
  __shared__ float tops[4];
  __shared__ double roots[kRootCount];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, slice = blockIdx.x, V = a.vocab;
  if (tid < kRootCount) roots[tid] = kRoots[tid];
  const Settings s = draw_settings(a, row);
  Four raw[E];
  slice_fetch<E>(a.logits + (int64_t)row * V, slice * 1024 * E, V, tid, -INFINITY, raw);
  if (LIMITS)
    for (int i = tid; i < kCopies * kBins; i += 256) {
      mass[i] = 0;
      if (COUNT) count[i] = 0;
    }
  float x[4 * E], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4 * E; ++i) {
    x[i] = draw_clean(raw[i / 4].v[i % 4]);
    top = fmaxf(top, x[i]);
  }
  top = wave_top(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const int best = draw_bin(top, s.grid);
  const int copy = (tid & (kCopies - 1)) * kBins;
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 4 * E; ++i) {
    const double w = draw_weight(x[i], top, s.scale, roots);
    sum += w;
    if (LIMITS && x[i] > -INFINITY) {
      const int j = min(best - draw_bin(x[i], s.grid), kBins - 1);
      atomicAdd(&mass[copy + j], scan_fix(w));
      if (COUNT) atomicAdd(&count[copy + j], 1u);
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  const int64_t at = (int64_t)row * a.slices + slice;
  if (tid == 0) {
    a.stat[at] = SliceStat{top, best, top > -INFINITY ? (sums[0] + sums[1]) + (sums[2] + sums[3]) : 0.0};
    if (LIMITS && slice == 0) a.listed[row] = 0;
  }
  static_assert(kBins == 256, "a bin a thread");
  if (LIMITS) {
    a.mass[at * kBins + tid] = scan_sum(mass + tid);
    if (COUNT) {
      uint32_t c = 0;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) c += count[i * kBins + tid];
      a.count[at * kBins + tid] = c;
    }
  }
}

// One wave: mass and count [kBins] become sums up to each bin, four a lane (total: the whole row's weight at least); where
// the borders lie.
template <bool COUNT>
__device__ __forceinline__ RowPlan draw_plan(double* mass, int* count, double total, float top, int bin,
                                             const Settings& s, int lane) {
  double b[4], upto[4];
  int d[4] = {0, 0, 0, 0}, cs[4] = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    b[k] = mass[4 * lane + k];
    if (COUNT) d[k] = count[4 * lane + k];
  }
  const double sum = wave_scan((b[0] + b[1]) + (b[2] + b[3]));
  upto[0] = sum - ((b[0] + b[1]) + (b[2] + b[3])) + b[0];
#pragma unroll
  for (int k = 1; k < 4; ++k) upto[k] = upto[k - 1] + b[k];
  if (lane == 63) upto[3] = fmax(total, upto[3]);
  if (COUNT) {
    cs[0] = wave_scan(d[0] + d[1] + d[2] + d[3]) - d[1] - d[2] - d[3];
#pragma unroll
    for (int k = 1; k < 4; ++k) cs[k] = cs[k - 1] + d[k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    mass[4 * lane + k] = upto[k];
    if (COUNT) count[4 * lane + k] = cs[k];
  }
  total = last_lane(upto[3]);
  // the first bin up to which the sum is not below x (the last one if there is none)
  auto first_at = [&](bool b0, bool b1, bool b2, bool b3) {
    const unsigned long long who = __ballot(b0 || b1 || b2 || b3);
    if (!who) return kBins - 1;
    const int at = __ffsll((long long)who) - 1, mine = b0 ? 0 : b1 ? 1 : b2 ? 2 : 3;
    return 4 * at + __builtin_amdgcn_readlane(mine, at);
  };
  auto first_sum = [&](double x) { return first_at(upto[0] >= x, upto[1] >= x, upto[2] >= x, upto[3] >= x); };
  RowPlan p{top, -INFINITY, 0.0f, 0.0f, 0.0f, 0.0f, bin, kBins, -1, kBins, 0, 0.0, 0.0, total};
  if (top > -INFINITY) {
    int b1 = kBins;                                    // where top_k's or min_p's border lies
    if (s.k == 1) b1 = 0;
    else if (COUNT && s.k > 0) b1 = first_at(cs[0] >= s.k, cs[1] >= s.k, cs[2] >= s.k, cs[3] >= s.k);
    if (s.min_p > 0.0f && s.min_p <= 1.0f) {
      // the least logit with (x - top) / T >= ln min_p: an estimate, then its neighbours
      const double z = log((double)s.min_p);
      auto in = [&](float x) { return ((double)x - (double)top) * s.inv_t >= z; };
      float xm = (float)((double)top + z / s.inv_t);
      if (!(xm > -FLT_MAX)) xm = -FLT_MAX;
      if (xm > top) xm = top;
      for (int i = 0; i < 4 && xm > -FLT_MAX && in(unordered(ordered(xm) - 1)); ++i) xm = unordered(ordered(xm) - 1);
      for (int i = 0; i < 4 && xm < top && !in(xm); ++i) xm = unordered(ordered(xm) + 1);
      p.xm = xm;
      const long long down = (long long)bin - draw_bin(xm, s.grid);
      b1 = min(b1, (int)min(down, (long long)(kBins - 1)));
    }
    p.limit = b1;
    p.first = b1;
    p.last = b1 < kBins ? b1 : -1;
    if (b1 > 0 && b1 < kBins) {
      if (COUNT) p.count1 = count[b1 - 1];
      p.mass1 = mass[b1 - 1];
    }
    if (s.p < 1.0f) {
      // the weight of what top_k and min_p keep lies between that of the bins before theirs and with it
      const double least = b1 == kBins ? total : p.mass1, most = b1 == kBins ? total : mass[b1];
      const double goal0 = (double)s.p * least, goal1 = (double)s.p * most;
      p.first = min(first_sum(goal0), b1);
      p.last = min(first_sum(goal1), b1);
    }
    if (p.first > 0) p.mass0 = mass[p.first - 1];
  }
  return p;
}

// The least logit of the bins up to `down` below bin (NaN: there is none): a search among the keys, 64 parts at a time, by
// one wave.
__device__ __forceinline__ float draw_edge(int down, int bin, float grid, int lane) {
  if (down < 0) return __uint_as_float(0x7FC00000u);
  if (down >= kBins - 1) return -FLT_MAX;
  uint32_t lo = ordered(-FLT_MAX), span = ordered(FLT_MAX) - lo;       // the border lies from lo to lo + span
  while (span > 0) {
    const uint32_t step = span / 64 + 1, k = lo + min((uint32_t)(lane + 1) * step - 1, span);
    const unsigned long long in = __ballot(draw_bin(unordered(k), grid) >= bin - down);
    const int at = __ffsll((long long)in) - 1;           // the row's largest logit is in: there is one
    lo += (uint32_t)at * step;
    span = min(step - 1, span - (uint32_t)at * step);
  }
  return unordered(lo);
}

template <bool COUNT>
struct PlanShared {
  double mass[kBins], factor[64], roots[kRootCount];
  int count[COUNT ? kBins : 1], offset[64];
  float tops[4], edges[4];
  RowPlan plan;
};

// The row's plan into sh.plan, by a work group of 256; fetch() is called when the loads of the bins are on their way.
template <bool COUNT, typename F>
__device__ __forceinline__ void draw_row_plan(const DrawArgs& a, int row, PlanShared<COUNT>& sh, int tid, F fetch) {
  const int lane = tid & 63, wave = tid >> 6;
  if (tid < kRootCount) sh.roots[tid] = kRoots[tid];
  const Settings s = draw_settings(a, row);
  const SliceStat* stat = a.stat + (int64_t)row * a.slices;
  const int j = tid;                                     // this thread's bin
  float top = -INFINITY;
  for (int i = tid; i < a.slices; i += 256) top = fmaxf(top, stat[i].top);
  top = wave_top(top);
  if (lane == 0) sh.tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sh.tops[0], sh.tops[1]), fmaxf(sh.tops[2], sh.tops[3]));
  const int bin = draw_bin(top, s.grid);
  // The row's bins, 64 slices at a time: thread j takes what falls on bin j; the last bin has the rest
  double m = 0.0, total = 0.0;
  int c = 0;
  for (int s0 = 0; s0 < a.slices; s0 += 64) {
    const int n = min(64, a.slices - s0);
    __syncthreads();
    if (wave == 0) {
      const SliceStat t = stat[s0 + (lane < n ? lane : 0)];
      const bool any = lane < n && t.top > -INFINITY;
      const double f = any ? draw_weight(t.top, top, s.scale, sh.roots) : 0.0;
      sh.factor[lane] = f * (1.0 / kSliceUnit);
      sh.offset[lane] = any ? bin - t.bin : kBins;       // 0 or more; nothing of an empty slice
      total += wave_sum(any ? f * t.sum : 0.0);
    }
    __syncthreads();
    const unsigned long long* at = a.mass + ((int64_t)row * a.slices + s0) * kBins;
    const uint32_t* ct = a.count + ((int64_t)row * a.slices + s0) * kBins;
    unsigned long long v[8];
    uint32_t cv[8];
    for (int i0 = 0; i0 < n; i0 += 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = min(i0 + k, n - 1), where = i * kBins + max(j - sh.offset[i], 0);
        v[k] = at[where];
        cv[k] = COUNT ? ct[where] : 0u;
      }
      if (s0 == 0 && i0 == 0) {
        // behind the bins: loads return in order
        __builtin_amdgcn_sched_barrier(0);
        fetch();
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (i0 + k < n && j >= sh.offset[i0 + k] && j < kBins - 1) {
          m += sh.factor[i0 + k] * (double)v[k];
          if (COUNT) c += (int)cv[k];
        }
    }
  }
  sh.mass[j] = m;
  if (COUNT) sh.count[j] = c;
  __syncthreads();
  if (wave == 0) {
    const RowPlan p = draw_plan<COUNT>(sh.mass, sh.count, total, top, bin, s, lane);
    if (lane == 0) sh.plan = p;
  }
  __syncthreads();
  // the bins' borders as logits, one a wave
  const int first = sh.plan.first, last = sh.plan.last, limit = sh.plan.limit;
  sh.edges[wave] = draw_edge(wave == 0 ? first - 1 : wave == 1 ? last : wave == 2 ? limit - 1 : limit, bin, s.grid, lane);
  __syncthreads();
  if (tid == 0) {
    sh.plan.x_first = sh.edges[0];
    sh.plan.x_last = sh.edges[1];
    sh.plan.x_before = sh.edges[2];
    sh.plan.x_limit = sh.edges[3];
  }
  __syncthreads();
}

// The plans of rows by a work group each, for k_draw_list with long slices, of which there are many: formed by each of
// its work groups they cost more than this launch (128 x 128256 with top_k and top_p 34 us, 7 + 16 with it; 64 rows with top_p
// 17, 6 + 13).
template <bool COUNT>
__global__ void __launch_bounds__(256) k_draw_plan(DrawArgs a) {
  __shared__ PlanShared<COUNT> sh;
  draw_row_plan<COUNT>(a, blockIdx.x, sh, threadIdx.x, []() {});
  if (threadIdx.x == 0) a.plan[blockIdx.x] = sh.plan;
}

template <int E, bool COUNT>
__global__ void __launch_bounds__(256, 4) k_draw_list(DrawArgs a) {
  constexpr bool PLANNED = plan_first(E);
  __shared__ PlanShared<COUNT && !PLANNED> sh;
  __shared__ unsigned long long parts[4];
  __shared__ int counts[4], base;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, slice = blockIdx.x, V = a.vocab;
  const SliceStat own = a.stat[(int64_t)row * a.slices + slice];
  const int j = tid;                                     // this thread's bin
  const unsigned long long own_mass = a.mass[((int64_t)row * a.slices + slice) * kBins + j];
  Four raw[E];                                           // on its way while the borders are found
  auto fetch = [&]() __attribute__((always_inline)) {
    slice_fetch<E>(a.logits + (int64_t)row * V, slice * 1024 * E, V, tid, -INFINITY, raw);
  };
  if constexpr (PLANNED) {
    fetch();
  } else {
    draw_row_plan<COUNT>(a, row, sh, tid, fetch);
    if (tid == 0 && slice == 0) a.plan[row] = sh.plan;
  }
  const RowPlan& plan = PLANNED ? a.plan[row] : sh.plan;
  const int first = plan.first, last = plan.last, limit = plan.limit, bin = plan.bin;
  const float hi1 = plan.x_first, lo1 = plan.x_last, hi2 = plan.x_before, lo2 = plan.x_limit;
  // this slice's weights in the bins before first
  if (first < kBins) {
    unsigned long long w = bin - own.bin + j < first && own.top > -INFINITY ? own_mass : 0;
    w = wave_sum(w);
    if (lane == 0) parts[wave] = w;
    __syncthreads();
    if (tid == 0) a.sure[(int64_t)row * a.slices + slice] = (double)((parts[0] + parts[1]) + (parts[2] + parts[3])) * (1.0 / kSliceUnit);
  } else if (tid == 0) {
    a.sure[(int64_t)row * a.slices + slice] = own.sum;
  }
  if (first > last) return;
  if (!(own.top > -INFINITY) || min(bin - own.bin, kBins - 1) > (limit < kBins ? limit : last)) return;
  uint32_t mine = 0;                                     // which of them are listed
  const bool two = limit > last && limit < kBins;
  auto within = [](float v, float lo, float hi) __attribute__((always_inline)) { return v >= lo && !(v >= hi); };
#pragma unroll
  for (int i = 0; i < 4 * E; ++i)
    if (within(raw[i / 4].v[i % 4], lo1, hi1)) mine |= 1u << i;
  if (two)
#pragma unroll
    for (int i = 0; i < 4 * E; ++i)
      if (within(raw[i / 4].v[i % 4], lo2, hi2)) mine |= 1u << i;
  const int n = __popc(mine), upto = wave_scan(n);
  if (lane == 63) counts[wave] = upto;
  __syncthreads();
  if (tid == 0) {
    const int all = counts[0] + counts[1] + counts[2] + counts[3];
    base = all ? atomicAdd(&a.listed[row], all) : 0;
  }
  __syncthreads();
  int at = base + upto - n;
  for (int w = 0; w < wave; ++w) at += counts[w];
  unsigned long long* list = a.list + (int64_t)row * kList;
#pragma unroll
  for (int i = 0; i < 4 * E; ++i)
    if (mine >> i & 1u) {
      if (at < kList) list[at] = draw_key(draw_clean(raw[i / 4].v[i % 4]), slice * 1024 * E + 1024 * (i / 4) + 4 * tid + i % 4);
      ++at;
    }
}

template <int NT>
struct BorderShared {
  unsigned long long pm[NT], ull[3][NT / 64], before_mass;
  uint32_t pc[NT];
  int ints[NT / 64], part, part_count, before_count;
};

// The least kept key among the n listed ones (key_at; 0: none there): by the whole work group of NT threads.
template <int NT, typename K>
__device__ __forceinline__ unsigned long long draw_border(const RowPlan& p, const Settings& s, double unit,
                                                          const double* roots, int n, K key_at, BorderShared<NT>& sh,
                                                          int tid) {
  // Keys at a time in a part's sums: the operations of four weights overlap, where lists are long
  constexpr int NW = NT / 64, AT = NT >= 512 ? 4 : 1;
  const int lane = tid & 63, wave = tid >> 6;
  // the least key of bins first .. last and the greatest of bin limit; the greatest of all
  unsigned long long low = ~0ull, most = 0, high = 0;
#pragma unroll 1
  for (int i = tid; i < n; i += NT) {
    const unsigned long long k = key_at(i);
    if (!k) continue;
    low = min(low, k);
    high = max(high, k);
    if (min(p.bin - draw_bin(key_logit(k), s.grid), kBins - 1) == p.limit) most = max(most, k);
  }
  auto greater = [](unsigned long long x, unsigned long long y) __attribute__((always_inline)) { return max(x, y); };
  auto lesser = [](unsigned long long x, unsigned long long y) __attribute__((always_inline)) { return min(x, y); };
  low = last_lane(wave_fold(low, ~0ull, lesser));
  high = last_lane(wave_fold(high, 0ull, greater));
  most = last_lane(wave_fold(most, 0ull, greater));
  if (lane == 0) {
    sh.ull[0][wave] = low;
    sh.ull[1][wave] = high;
    sh.ull[2][wave] = most;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    low = min(low, sh.ull[0][w]);
    high = max(high, sh.ull[1][w]);
    most = max(most, sh.ull[2][w]);
  }
  unsigned long long least = 0;
  if (p.limit < kBins && p.xm > -INFINITY) least = (unsigned long long)ordered(p.xm) << 32;
  // First where top_k ends (in bin limit), then where top_p does: of the keys from lo to hi in falling order, the one
  // at which the count from have on reaches want, or the weight from sum on reaches goal.
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {
    const bool counting = stage == 0;
    if (counting ? !(p.limit < kBins && s.k > 0) : !(s.p < 1.0f)) continue;
    unsigned long long lo = least, hi = most, sum = 0;
    int have = p.count1;
    double goal = 0.0;
    if (!counting) {
      double of = p.total;
      if (p.limit < kBins) {                         // what top_k and min_p keep
        unsigned long long w = 0;
#pragma unroll 1
        for (int i = tid; i < n; i += NT) {
          const unsigned long long k = key_at(i);
          if (k && k >= least && k <= most) w += list_fix(draw_weight(key_logit(k), p.top, s.scale, roots), unit);
        }
        w = wave_sum(w);
        __syncthreads();
        if (lane == 0) sh.ull[0][wave] = w;
        __syncthreads();
        w = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) w += sh.ull[0][i];
        of = (double)w / unit + p.mass1;
      }
      goal = (double)s.p * of * unit;
      sum = (unsigned long long)(p.mass0 * unit);
      // the border lies in bins first .. last; between them and bin limit lie tokens that are not listed
      if (p.last < p.limit) lo = max(max(lo, most + 1), (unsigned long long)ordered(p.x_last) << 32);
      hi = high;
      least = lo;
    }
    lo = max(lo, low);
    if (lo > hi) {                                   // there are none: what lies before
      least = counting ? least : (unsigned long long)ordered(p.x_first) << 32;
      continue;
    }
    while (lo < hi) {
      const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - (NT == 512 ? 9 : 8));
      __syncthreads();
      sh.pm[tid] = 0;
      sh.pc[tid] = 0;
      if (tid == 0) sh.part = INT32_MAX;
      __syncthreads();
#pragma unroll 1
      for (int i = tid; i < n; i += AT * NT) {
        unsigned long long k[AT];
        bool in[AT], any = false;
#pragma unroll
        for (int j = 0; j < AT; ++j) {
          k[j] = i + j * NT < n ? key_at(i + j * NT) : 0ull;
          in[j] = k[j] && k[j] >= lo && k[j] <= hi;
          any |= in[j];
        }
        if (!any) continue;
        unsigned long long w[AT];
        if (!counting)
#pragma unroll
          for (int j = 0; j < AT; ++j) w[j] = list_fix(draw_weight(key_logit(k[j]), p.top, s.scale, roots), unit);
#pragma unroll
        for (int j = 0; j < AT; ++j)
          if (in[j]) {
            const int at = NT - 1 - (int)((k[j] - lo) >> shift);       // falling
            atomicAdd(&sh.pc[at], 1u);
            if (!counting) atomicAdd(&sh.pm[at], w[j]);
          }
      }
      __syncthreads();
      const unsigned long long m0 = sh.pm[tid], ms = wave_scan(m0);
      const int c0 = (int)sh.pc[tid], cs = wave_scan(c0);
      if (lane == 63) {
        sh.ull[0][wave] = ms;
        sh.ints[wave] = cs;
      }
      __syncthreads();
      unsigned long long me = ms;
      int ce = cs;
#pragma unroll
      for (int w = 0; w < NW; ++w)
        if (w < wave) {
          me += sh.ull[0][w];
          ce += sh.ints[w];
        }
      const bool there = c0 && (counting ? have + ce >= s.k : (double)(sum + me) >= goal);
      const unsigned long long who = __ballot(there);
      if (who && lane == __ffsll((long long)who) - 1) atomicMin(&sh.part, tid);
      __syncthreads();
      const int at = sh.part;
      if (at == INT32_MAX) break;                    // not reached: all of them
      if (at == tid) {                               // what lies before that part
        sh.before_count = ce - c0;
        sh.before_mass = me - m0;
        sh.part_count = c0;
      }
      __syncthreads();
      have += sh.before_count;
      sum += sh.before_mass;
      const unsigned long long from = lo + ((unsigned long long)(NT - 1 - at) << shift);
      const unsigned long long to = from + ((1ull << shift) - 1);
      lo = max(lo, from);
      hi = min(hi, to);
      if (sh.part_count == 1) break;                    // the only key from lo to hi
    }
    least = lo;
  }
  // A border among the keys of -0, which no logit has: all zeros lie above it (compared as numbers, they would equal it and
  // be kept by their index)
  if ((uint32_t)(least >> 32) == ordered(-0.0f)) least = (unsigned long long)ordered(0.0f) << 32;
  return least;
}

// The token among a slice's kept weights (raw: its logits from `from` on, pass after pass of four a thread; weight(x, t): 0 if it
// is not kept): the first whose sum passes want, the last with any where rounding leaves none.  WHOLE: want is a
// share of the slice's sum, whose logarithm is taken here; else log_kept is the logarithm of the row's kept weights.  Passes
// stay a loop, and the waves' sums of all passes are gone through at once: one barrier, and code that is run
// once is short (it comes from memory).  256 x 32000 without limits 16.2 -> 14.6 us, 512 x 1000 6.8 -> 4.7.
template <int NT, int NP, bool WHOLE, typename F>
__device__ __forceinline__ void draw_token(const DrawArgs& a, int row, const Four (&raw)[NP], int from, float top,
                                           const Settings& s, float xb, double want, double log_kept, double* chunk,
                                           int tid, F weight) {
  constexpr int NW = NT / 64, PASS = 4 * NT;
  static_assert(NP * NW <= 64, "a lane a sum");
  const int lane = tid & 63, wave = tid >> 6;
  double part[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) part[k] = 0.0;
#pragma unroll 1
  for (int i = 0; i < NP; ++i) {
    Four f = raw[0];                                       // raw[i], without an index into registers
#pragma unroll
    for (int k = 1; k < NP; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = i == k ? raw[k].v[j] : f.v[j];
    double w = 0.0;
    const float most = fmaxf(fmaxf(f.v[0], f.v[1]), fmaxf(f.v[2], f.v[3]));
    if (__ballot(draw_clean(most) >= xb))
#pragma unroll
      for (int j = 0; j < 4; ++j) w += weight(draw_clean(f.v[j]), from + PASS * i + 4 * tid + j);
#pragma unroll
    for (int k = 0; k < NP; ++k) part[k] = i == k ? w : part[k];
    w = wave_sum(w);
    if (lane == 0) chunk[i * NW + wave] = w;
  }
  __syncthreads();
  // the place up to which the sums pass want; before: what lies before it
  auto place = [&](double w, double c, double& before) __attribute__((always_inline)) {
    const unsigned long long over = __ballot(w > 0.0 && c > want), any = __ballot(w > 0.0);
    const int at = over ? __ffsll((long long)over) - 1 : any ? 63 - __clzll((long long)any) : -1;
    before = __shfl(c - w, max(at, 0), 64);
    return at;
  };
  const double w = lane < NP * NW ? chunk[lane] : 0.0, c = wave_scan(w);
  if (WHOLE) {
    const double all = last_lane(c);
    want *= all;
    log_kept = ln_of(all);
  }
  double before;
  const int at = __builtin_amdgcn_readfirstlane(place(w, c, before));
  if (at < 0) {                                            // cannot be: the slice has weight
    if (tid == 0) a.tokens[row] = from;
    return;
  }
  if (wave != at % NW) return;
  Four f = raw[0];
  double mine = part[0];
#pragma unroll
  for (int i = 1; i < NP; ++i) {
    const bool it = i == at / NW;
    mine = it ? part[i] : mine;
#pragma unroll
    for (int j = 0; j < 4; ++j) f.v[j] = it ? raw[i].v[j] : f.v[j];
  }
  want -= before;
  const int who = place(mine, wave_scan(mine), before);
  if (lane != who) return;
  const int t0 = from + PASS * (at / NW) + 4 * tid;
  double sum = before;
  int token = -1, last = t0;
  float x = 0.0f, last_x = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float v = draw_clean(f.v[j]);
    const double one = weight(v, t0 + j);
    sum += one;
    if (one > 0.0) {
      last = t0 + j;
      last_x = v;
      if (sum > want && token < 0) {
        token = last;
        x = v;
      }
    }
  }
  if (token < 0) {
    token = last;
    x = last_x;
  }
  a.tokens[row] = token;
  if (a.logprobs) a.logprobs[row] = s.best ? 0.0f : (float)(((double)x - (double)top) * s.inv_t - log_kept);
}

constexpr int kMaxSlices = 2048;

// What bounds a row is its chain of barriers, so short slices take few waves (one row of 32003: 9.0 us, 10.3 with 512 threads
// and 12.5 with 1024); long ones 512 threads (128 x 128256: 19.4 us, 19.8 with 1024).
constexpr int pick_threads(bool limits, int E) { return limits && E > 2 ? 512 : 256; }

template <bool LIMITS, int E>
__global__ void __launch_bounds__(pick_threads(LIMITS, E)) k_draw_pick(DrawArgs a) {
  constexpr int NT = pick_threads(LIMITS, E), NW = NT / 64, SLICE = 1024 * E;
  __shared__ unsigned long long keys[LIMITS ? kList : 1], add[LIMITS ? kMaxSlices : 1];
  __shared__ BorderShared<LIMITS ? NT : 64> sh;
  __shared__ double chunk[SLICE / 256];
  __shared__ float tops[NW];
  __shared__ int slice_at;
  __shared__ double before_slice, all_kept;
  __shared__ double roots[kRootCount];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x, V = a.vocab;
  if (tid < kRootCount) roots[tid] = kRoots[tid];
  const float* x = a.logits + (int64_t)row * V;
  const SliceStat* stat = a.stat + (int64_t)row * a.slices;
  const SliceStat first_stat = stat[lane < a.slices ? lane : 0];       // on their way
  const double first_sure = LIMITS ? a.sure[(int64_t)row * a.slices + (lane < a.slices ? lane : 0)] : 0.0;
  const Settings s = draw_settings(a, row);
  float u = a.uniforms[row];
  const bool bad = s.bad || !(u >= 0.0f && u < 1.0f);
  u = u >= 1.0f ? 1.0f - 0x1p-24f : u > 0.0f ? u : 0.0f;
  if (bad && tid == 0) atomicOr(a.err, kErrSample);
  if (!LIMITS && s.best) u = 0.0f;                       // the first of the best
  __shared__ RowPlan plan;
  const RowPlan& p = plan;                               // in LDS
  int n_list = 0;
  if (LIMITS) {
    if (tid == 0) plan = a.plan[row];
    n_list = a.listed[row];
    __syncthreads();
  } else {
    float top = -INFINITY;
    for (int i = tid; i < a.slices; i += NT) top = fmaxf(top, stat[i].top);
    top = wave_top(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, tops[w]);
    if (tid == 0) {
      plan = RowPlan{};
      plan.top = top;
      plan.first = kBins;
      plan.last = -1;
    }
    __syncthreads();
  }
  if (!(p.top > -INFINITY)) {                            // nothing to draw
    if (tid == 0) {
      a.tokens[row] = -1;
      if (a.logprobs) a.logprobs[row] = -INFINITY;
    }
    return;
  }
  auto bin_of = [&](float v) __attribute__((always_inline)) { return min(p.bin - draw_bin(v, s.grid), kBins - 1); };
  const double unit = LIMITS ? list_unit(p.total) : 1.0;
  auto fixed = [&](unsigned long long k) __attribute__((always_inline)) {
    return list_fix(draw_weight(key_logit(k), p.top, s.scale, roots), unit);
  };

  unsigned long long border = draw_key(-FLT_MAX, INT32_MAX);           // keys from here on are kept
  if constexpr (LIMITS) {
    for (int i = tid; i < a.slices; i += NT) add[i] = 0;
    if (p.first <= p.last) {
      // The listed keys (no key is 0): in LDS, or taken from the row each time where the list did not hold them.
      // Loops stay loops: unrolled, this kernel was 40 KB of code, which it waited for.
      const bool held = n_list <= kList;
      const int n = held ? n_list : V;
      const unsigned long long* list = a.list + (int64_t)row * kList;
      auto from_row = [&](int t) {
        const float v = draw_clean(x[t]);
        const int b = bin_of(v);
        return v > -INFINITY && ((b >= p.first && b <= p.last) || b == p.limit) ? draw_key(v, t) : 0ull;
      };
      if (held) {
#pragma unroll 4
        for (int i = tid; i < n; i += NT) keys[i] = list[i];
        __syncthreads();
      }
      auto key_at = [&](int i) __attribute__((always_inline)) { return held ? keys[i] : from_row(i); };
      border = max(border, draw_border<NT>(p, s, unit, roots, n, key_at, sh, tid));
      // the listed tokens' share of their slices
      __syncthreads();
#pragma unroll 1
      for (int i = tid; i < n; i += NT) {
        const unsigned long long k = key_at(i);
        if (k && k >= border) atomicAdd(&add[key_token(k) / SLICE], fixed(k));
      }
    }
    __syncthreads();
  }
  // kept: logits above xb, and those equal to it up to token tb
  const float least = draw_floor(p.top, s), border_x = LIMITS ? key_logit(border) : s.best ? p.top : -FLT_MAX;
  const float xb = fmaxf(border_x, least);
  const uint32_t tb = LIMITS && border_x >= least ? (uint32_t)key_token(border) : UINT32_MAX;
  auto kept = [&](float v, int t) __attribute__((always_inline)) { return v > xb || (v == xb && (uint32_t)t <= tb); };
  // The slices' kept weights, summed up in their order by one wave; the first whose sum passes u times the whole (the
  // last one with any where rounding leaves none)
  if (wave == 0) {
    const double* own = LIMITS ? a.sure + (int64_t)row * a.slices : nullptr;
    auto of = [&](int i, const SliceStat& t, double sure) __attribute__((always_inline)) {
      if (i >= a.slices) return 0.0;
      if (!(t.top > -INFINITY)) return 0.0;
      if (!LIMITS && s.best) return t.top == p.top ? 1.0 : 0.0;
      if (t.top < least) return 0.0;
      double w = draw_weight(t.top, p.top, s.scale, roots) * (LIMITS ? sure : t.sum);
      if (LIMITS) w += (double)add[i] / unit;
      return w;
    };
    double run = 0.0;
    auto later = [&](int i) {
      const int k = i < a.slices ? i : 0;
      return of(i, stat[k], LIMITS ? own[k] : 0.0);
    };
    const double w0 = of(lane, first_stat, first_sure);
    for (int s0 = 0; s0 < a.slices; s0 += 64) run += wave_sum(s0 ? later(s0 + lane) : w0);
    const double target = (double)u * run;
    double upto = 0.0, before = 0.0;
    int found = -1;
    for (int s0 = 0; s0 < a.slices; s0 += 64) {
      const double w = s0 ? later(s0 + lane) : w0, c = upto + wave_scan(w);
      const unsigned long long over = __ballot(w > 0.0 && c > target), any = __ballot(w > 0.0);
      if (any) {
        const int at = over ? __ffsll((long long)over) - 1 : 63 - __clzll((long long)any);
        const double b = __shfl(c - w, at, 64);
        found = s0 + at;
        before = b;
      }
      if (over) break;
      upto = last_lane(c);
    }
    if (lane == 0) {
      slice_at = max(found, 0);
      before_slice = before;
      all_kept = run;
    }
  }
  __syncthreads();
  // the token in that slice
  const int from = slice_at * SLICE;
  Four raw[SLICE / (4 * NT)];
  slice_fetch<SLICE / (4 * NT), 4 * NT>(x, from, V, tid, -INFINITY, raw);
  __builtin_amdgcn_sched_barrier(0);
  const double log_kept = ln_of(all_kept);                 // while they are on their way
  draw_token<NT, SLICE / (4 * NT), false>(a, row, raw, from, p.top, s, xb, (double)u * all_kept - before_slice, log_kept,
                                          chunk, tid, [&](float v, int k) __attribute__((always_inline)) {
                                            return kept(v, k) ? draw_weight(v, p.top, s.scale, roots) : 0.0;
                                          });
}

// The whole draw of a row of up to 4 NT E logits by one work group, which holds them in registers: the same steps with
// the row for a slice, one launch and no memory in between: 512 rows of 1000 47 -> 13 us, one row of 1000 19 -> 10.5, 256 of
// 8192 27 -> 20; from 16384 on the slices are faster (one row 20 against 27 us).  Few waves, for the barriers.
template <bool LIMITS, bool COUNT, int NT, int E>
__global__ void __launch_bounds__(NT) k_draw_row(DrawArgs a) {
  constexpr int NW = NT / 64, PASS = 4 * NT;
  __shared__ unsigned long long keys[LIMITS ? PASS * E : 1], bins[LIMITS ? kCopies * kBins : 1];
  __shared__ uint32_t counts[COUNT ? kCopies * kBins : 1];
  __shared__ BorderShared<LIMITS ? NT : 64> sh;
  __shared__ double mass[kBins], chunk[E * NW], roots[kRootCount];
  __shared__ int count[kBins];
  __shared__ float tops[NW], edges[4];
  __shared__ RowPlan plan;
  __shared__ int n_list;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x, V = a.vocab;
  if (tid < kRootCount) roots[tid] = kRoots[tid];
  const float* x = a.logits + (int64_t)row * V;
  Four raw[E];
  slice_fetch<E, PASS>(x, 0, V, tid, -INFINITY, raw);
  const Settings s = draw_settings(a, row);
  float u = a.uniforms[row];
  const bool bad = s.bad || !(u >= 0.0f && u < 1.0f);
  u = u >= 1.0f ? 1.0f - 0x1p-24f : u > 0.0f ? u : 0.0f;
  if (bad && tid == 0) atomicOr(a.err, kErrSample);
  if (!LIMITS && s.best) u = 0.0f;                       // the first of the best
  if (LIMITS)
    for (int i = tid; i < kCopies * kBins; i += NT) {
      bins[i] = 0;
      if (COUNT) counts[i] = 0;
    }
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      raw[i].v[j] = draw_clean(raw[i].v[j]);
      top = fmaxf(top, raw[i].v[j]);
    }
  top = wave_top(top);
  if (lane == 0) tops[wave] = top;
  if (tid == 0) n_list = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, tops[w]);
  if (!(top > -INFINITY)) {                              // nothing to draw
    if (tid == 0) {
      a.tokens[row] = -1;
      if (a.logprobs) a.logprobs[row] = -INFINITY;
    }
    return;
  }
  unsigned long long border = draw_key(-FLT_MAX, INT32_MAX);           // keys from here on are kept
  if constexpr (LIMITS) {
    const int bin = draw_bin(top, s.grid), copy = (tid & (kCopies - 1)) * kBins;
#pragma unroll
    for (int i = 0; i < 4 * E; ++i) {
      const float v = raw[i / 4].v[i % 4];
      if (v > -INFINITY) {
        const int j = min(bin - draw_bin(v, s.grid), kBins - 1);
        atomicAdd(&bins[copy + j], scan_fix(draw_weight(v, top, s.scale, roots)));
        if (COUNT) atomicAdd(&counts[copy + j], 1u);
      }
    }
    __syncthreads();
    if (tid < kBins) {
      mass[tid] = (double)scan_sum(bins + tid) * (1.0 / kSliceUnit);
      if (COUNT) {
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) c += counts[i * kBins + tid];
        count[tid] = (int)c;
      }
    }
    __syncthreads();
    if (wave == 0) {
      const RowPlan p = draw_plan<COUNT>(mass, count, 0.0, top, bin, s, lane);
      if (lane == 0) plan = p;
    }
    __syncthreads();
    const int first = plan.first, last = plan.last, limit = plan.limit;
    if (first <= last) {
      if (wave < 4)
        edges[wave] = draw_edge(wave == 0 ? first - 1 : wave == 1 ? last : wave == 2 ? limit - 1 : limit, bin, s.grid, lane);
      __syncthreads();
      const float hi1 = edges[0], lo1 = edges[1], hi2 = edges[2], lo2 = edges[3];
      const bool two = limit > last && limit < kBins;
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < 4 * E; ++i) {
        const float v = raw[i / 4].v[i % 4];
        if ((v >= lo1 && !(v >= hi1)) || (two && v >= lo2 && !(v >= hi2))) mine |= 1u << i;
      }
      const int n = __popc(mine), upto = wave_scan(n), all = last_lane(upto);
      int at = 0;
      if (lane == 0 && all) at = atomicAdd(&n_list, all);
      at = __builtin_amdgcn_readfirstlane(at) + upto - n;
#pragma unroll
      for (int i = 0; i < 4 * E; ++i)
        if (mine >> i & 1u) {
          keys[at++] = draw_key(raw[i / 4].v[i % 4], PASS * (i / 4) + 4 * tid + i % 4);
        }
      if (tid == 0) {
        plan.x_first = edges[0];
        plan.x_last = edges[1];
      }
      __syncthreads();
      const RowPlan& p = plan;                           // in LDS
      auto key_at = [&](int i) __attribute__((always_inline)) { return keys[i]; };
      border = max(border, draw_border<NT>(p, s, list_unit(p.total), roots, n_list, key_at, sh, tid));
    }
  }
  const float least = draw_floor(top, s), border_x = LIMITS ? key_logit(border) : s.best ? top : -FLT_MAX;
  const float xb = fmaxf(border_x, least);
  const uint32_t tb = LIMITS && border_x >= least ? (uint32_t)key_token(border) : UINT32_MAX;
  auto weight = [&](float v, int t) __attribute__((always_inline)) {
    return v > xb || (v == xb && (uint32_t)t <= tb) ? draw_weight(v, top, s.scale, roots) : 0.0;
  };
  draw_token<NT, E, true>(a, row, raw, 0, top, s, xb, (double)u, 0.0, chunk, tid, weight);
}

}  // namespace tmz

using namespace tmz;

namespace {

termezo_status refuse(termezo_ctx* c, const char* msg) {
  c->last_error = msg;
  return TERMEZO_ERR_INVALID_ARG;
}
termezo_status hip_status(termezo_ctx* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return TERMEZO_OK;
  (void)hipGetLastError();                               // reported here, not by the next launch
  c->last_error = std::string(what) + ": " + hipGetErrorString(e);
  return e == hipErrorOutOfMemory ? TERMEZO_ERR_OOM : TERMEZO_ERR_DEVICE;
}
bool words(std::initializer_list<const void*> ps) {      // 4-byte aligned (null is)
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) & 3u) return false;
  return true;
}

}  // namespace

extern "C" {

termezo_status termezo_adjust_logits(termezo_ctx* c, const float* logits, int32_t rows, int32_t vocab,
                                     const termezo_logit_rules* rules, float* out) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!logits || !rules || !out) return refuse(c, "adjust_logits: null pointer");
  const termezo_logit_rules& r = *rules;
  if (!words({logits, out, r.history, r.lengths, r.starts, r.repetition, r.presence, r.frequency, r.bias, r.bias_index,
              r.mask, r.mask_index}))
    return refuse(c, "adjust_logits: misaligned pointer");
  if (rows <= 0 || rows > 65535 || vocab <= 0 || vocab > (1 << 24) || r.hist_len < 0 || r.hist_len > (1 << 24))
    return refuse(c, "adjust_logits: a size is out of range");
  if ((r.bias_index && !r.bias) || (r.mask_index && !r.mask)) return refuse(c, "adjust_logits: indices without a table");
  if ((r.bias && (r.n_bias <= 0 || (!r.bias_index && r.n_bias != 1 && r.n_bias != rows))) ||
      (r.mask && (r.n_masks <= 0 || (!r.mask_index && r.n_masks != 1 && r.n_masks != rows))))
    return refuse(c, "adjust_logits: a table without lines, or without indices and lines neither 1 nor rows");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "adjust_logits");
  RuleArgs a{logits, out, vocab, r, c->d_err};
  if (a.r.hist_len == 0 && !r.lengths && !r.starts) a.r.history = nullptr;     // nothing to count, nothing to check
#define TMZ_ADJUST(SLICE, HIST)                                                                                    \
  hipLaunchKernelGGL((k_adjust<SLICE, HIST>), dim3((unsigned)((vocab + SLICE - 1) / SLICE), (unsigned)rows), dim3(256), 0, \
                     c->stream, a)
  const bool few = (int64_t)rows * ((vocab + 1023) / 1024) <= 4 * (int64_t)c->n_cu;
  if (a.r.history) {
    if (few) TMZ_ADJUST(1024, true);
    else TMZ_ADJUST(8192, true);
  } else {
    if (few) TMZ_ADJUST(1024, false);
    else TMZ_ADJUST(4096, false);
  }
#undef TMZ_ADJUST
  return hip_status(c, hipGetLastError(), "adjust_logits");
}

termezo_status termezo_sample(termezo_ctx* c, const float* logits, const float* uniforms, int32_t rows, int32_t vocab,
                              const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                              int32_t* tokens, float* logprobs) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!logits || !uniforms || !tokens) return refuse(c, "sample: null pointer");
  if (!words({logits, uniforms, temperature, top_k, top_p, min_p, tokens, logprobs}))
    return refuse(c, "sample: misaligned pointer");
  if (rows <= 0 || rows > 65535 || vocab <= 0 || vocab > (1 << 24)) return refuse(c, "sample: a size is out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "sample");
  const int64_t most = std::min<int64_t>(rows, kMaxDrawRows);      // rows at a time
  const bool limits = top_k || top_p || min_p;
  const bool whole = vocab <= 8192;      // a row by one work group
  const int long_slices = (vocab + 8191) / 8192;
  // Long slices where they give every compute unit two work groups: 256 x 32003 with top_p 46 us, 57 with short ones, 64 x
  // 128256 52 and 97; few rows are faster in short ones (one of 32003 20.4, 28.5 with long ones; 64 of them 32.4 and 33.4).
  // The grouping of a row's sums, and so their last bits, go with it.
  const bool large = (limits && most * long_slices >= 2 * (int64_t)c->n_cu) || long_slices > 64;
  const int slice = large ? 8192 : 2048, slices = (vocab + slice - 1) / slice;   // kMaxSlices at most
  const int64_t per_row = whole ? 0 : (int64_t)slices * sizeof(SliceStat) +
                          (limits ? (int64_t)slices * (kBins * 12 + 8) + sizeof(RowPlan) + 8 + (int64_t)kList * 8 : 0);
  const termezo_status st = scratch_for(c, c->draw, most * per_row, "sample");
  if (st != TERMEZO_OK) return st;
  DrawArgs a{};
  a.vocab = vocab;
  a.slices = slices;
  a.err = c->d_err;
  char* at = (char*)c->draw.p;
  auto take = [&](int64_t bytes) {
    char* p = at;
    at += bytes;
    return p;
  };
  a.stat = (SliceStat*)take(most * slices * sizeof(SliceStat));
  if (limits) {
    a.list = (unsigned long long*)take(most * kList * 8);
    a.mass = (unsigned long long*)take(most * slices * kBins * 8);
    a.sure = (double*)take(most * slices * 8);
    a.plan = (RowPlan*)take(most * sizeof(RowPlan));
    a.listed = (int32_t*)take(most * 8);
    a.count = (uint32_t*)take(most * slices * kBins * 4);
  }
  for (int r0 = 0; r0 < rows; r0 += kMaxDrawRows) {
    const int n = std::min(kMaxDrawRows, rows - r0);
    auto from = [&](auto* p) { return p ? p + r0 : p; };
    a.logits = logits + (int64_t)r0 * vocab;
    a.uniforms = uniforms + r0;
    a.temperature = from(temperature);
    a.top_k = from(top_k);
    a.top_p = from(top_p);
    a.min_p = from(min_p);
    a.tokens = tokens + r0;
    a.logprobs = from(logprobs);
    const dim3 grid((unsigned)slices, (unsigned)n);
    const dim3 rows_grid((unsigned)n);
    if (whole) {
#define TMZ_ROW(NT, E)                                                                                                 \
  if (!limits) hipLaunchKernelGGL((k_draw_row<false, false, NT, E>), rows_grid, dim3(NT), 0, c->stream, a);     \
  else if (top_k) hipLaunchKernelGGL((k_draw_row<true, true, NT, E>), rows_grid, dim3(NT), 0, c->stream, a);    \
  else hipLaunchKernelGGL((k_draw_row<true, false, NT, E>), rows_grid, dim3(NT), 0, c->stream, a)
      if (vocab <= 1024) {
        TMZ_ROW(256, 1);
      } else if (vocab <= 4096) {
        TMZ_ROW(256, 4);
      } else {
        TMZ_ROW(512, 4);
      }
#undef TMZ_ROW
      continue;
    }
#define TMZ_DRAW(E)                                                                                          \
  if (!limits) {                                                                                             \
    hipLaunchKernelGGL((k_draw_scan<E, false, false>), grid, dim3(256), 0, c->stream, a);                    \
    hipLaunchKernelGGL((k_draw_pick<false, E>), rows_grid, dim3(pick_threads(false, E)), 0, c->stream, a);                     \
  } else {                                                                                                   \
    if (top_k) {                                                                                             \
      hipLaunchKernelGGL((k_draw_scan<E, true, true>), grid, dim3(256), 0, c->stream, a);                    \
      if (plan_first(E)) hipLaunchKernelGGL((k_draw_plan<true>), rows_grid, dim3(256), 0, c->stream, a);     \
      hipLaunchKernelGGL((k_draw_list<E, true>), grid, dim3(256), 0, c->stream, a);                          \
    } else {                                                                                                 \
      hipLaunchKernelGGL((k_draw_scan<E, true, false>), grid, dim3(256), 0, c->stream, a);                   \
      if (plan_first(E)) hipLaunchKernelGGL((k_draw_plan<false>), rows_grid, dim3(256), 0, c->stream, a);    \
      hipLaunchKernelGGL((k_draw_list<E, false>), grid, dim3(256), 0, c->stream, a);                         \
    }                                                                                                        \
    hipLaunchKernelGGL((k_draw_pick<true, E>), rows_grid, dim3(pick_threads(true, E)), 0, c->stream, a);                      \
  }
    if (large) {
      TMZ_DRAW(8)
    } else {
      TMZ_DRAW(2)
    }
#undef TMZ_DRAW
  }
  return hip_status(c, hipGetLastError(), "sample");
}

}  // extern "C"
