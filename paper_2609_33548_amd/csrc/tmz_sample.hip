// From the logits to the next tokens: penalties, bias and allowed tokens, and the draw.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>

#include "tmz_device.h"
#include "tmz_internal.h"

namespace tmz {

constexpr int32_t kErrRules = 64, kErrSample = 128;      // bits of the deferred error word

struct __attribute__((packed, aligned(4))) Four {        // rows of any length begin at any multiple of 4 bytes
  float v[4];
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
  int32_t vocab, rows;
  termezo_logit_rules r;
  int32_t* err;
};

constexpr int kRuleSlice = 4096;

// Line of a table that row takes: -1 none.
__device__ __forceinline__ int rule_line(const int32_t* index, int lines, int row, bool& bad) {
  const int i = index ? index[row] : (lines == 1 ? 0 : row);
  if (i >= -1 && i < lines) return i;
  bad = true;
  return -1;
}

__global__ void __launch_bounds__(256) k_adjust(RuleArgs a) {
  __shared__ uint32_t count[kRuleSlice];
  const int tid = threadIdx.x, row = blockIdx.y, V = a.vocab;
  const int t0 = blockIdx.x * kRuleSlice, n = min(kRuleSlice, V - t0);
  bool bad = false;
  const bool hist = a.r.history != nullptr;
  float rep = 1.0f, freq = 0.0f, pres = 0.0f;
  if (hist) {
    for (int i = tid; i < n; i += 256) count[i] = 0u;
    int64_t len = a.r.hist_len, from = 0;
    if (a.r.lengths) {
      const int l = a.r.lengths[row];
      if (l < 0 || l > len) bad = true;
      len = bad ? 0 : l;
    }
    if (a.r.starts) {
      from = a.r.starts[row];
      if (from < 0 || (from > len && !bad)) {
        bad = true;
        len = 0;
      }
    }
    if (a.r.repetition) rep = a.r.repetition[row];
    if (a.r.frequency) freq = a.r.frequency[row];
    if (a.r.presence) pres = a.r.presence[row];
    __syncthreads();
    const int32_t* h = a.r.history + row * a.r.hist_len;
    for (int64_t i = tid; i < len; i += 256) {
      const uint32_t at = (uint32_t)h[i] - (uint32_t)t0;   // ids outside the vocabulary are outside every slice
      if (at < (uint32_t)n) {
        if (i >= from) atomicAdd(&count[at], 2u);
        else atomicOr(&count[at], 1u);
      }
    }
    __syncthreads();
  }
  const int bl = a.r.bias ? rule_line(a.r.bias_index, a.r.n_bias, row, bad) : -1;
  const int ml = a.r.mask ? rule_line(a.r.mask_index, a.r.n_masks, row, bad) : -1;
  if (bad && tid == 0 && blockIdx.x == 0) atomicOr(a.err, kErrRules);
  const float* x = a.logits + (int64_t)row * V;
  float* y = a.out + (int64_t)row * V;
  const float* bias = bl >= 0 ? a.r.bias + (int64_t)bl * V : nullptr;
  const uint32_t* mask = ml >= 0 ? a.r.mask + (int64_t)ml * ((V + 31) / 32) : nullptr;
  auto one = [&](float v, int i, float b, uint32_t allowed) __attribute__((always_inline)) {
    if (hist) {
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
// k_draw_scan, a work group for a slice of a row: the slice's largest logit m_s, its weights exp((x - m_s) / T)
// in fixed point (2^-48; integer sums do not depend on their order), their sum, and sums and counts by bins.
// A bin is a quarter of T wide on a grid that all slices share (bin = floor(x (4 / T))), counted from the slice's
// best bin downwards; the last of the 128 holds all that lies lower.
// k_draw_list, the same grid: the row's bins (slices weighted by exp((m_s - m) / T)) tell in which of them the
// borders lie; the slice's logits in those bins go to the row's list.
// k_draw_pick, a work group a row: finds the border in the list by narrowing a range of keys (logit, index) to
// 1024 parts at a time; then the slice and the token.  Where the list does not hold them (many equal logits)
// it goes through the row in the list's place.
// Without limits the first and the last are enough.
// ---------------------------------------------------------------------------
constexpr int kBins = 128, kList = 8192, kMaxDrawRows = 1024, kPickThreads = 512;
constexpr double kSliceUnit = 0x1p48;

struct SliceStat {
  float top;                         // -inf: nothing
  int32_t bin;
  unsigned long long sum;            // weights relative to top, 2^-48
};
struct RowPlan {                     // what k_draw_list found
  float top, xm;                     // the row's largest logit; the least one that min_p keeps
  int32_t bin;
  int32_t first, last;               // bins before first are kept, bins first .. last are listed
  int32_t limited;                   // whether top_k or min_p ends in the listed bins
  int32_t count0;                    // tokens and weight (relative to top) in the bins before first
  double mass0;
  double total;                      // of the whole row
};

struct DrawArgs {
  const float *logits, *uniforms, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens;
  float* logprobs;
  int32_t vocab, slices;
  SliceStat* stat;                   // [rows][slices]
  unsigned long long* mass;          // [rows][slices][kBins]
  uint32_t* count;
  RowPlan* plan;                     // [rows]
  int32_t* listed;                   // [rows]
  unsigned long long* list;          // [rows][kList]
  int32_t* err;
};

struct Settings {
  double inv_t;                      // 1 / T
  float grid;                        // 4 / T
  float p, min_p;                    // p 1: none; min_p 0: none
  int k;                             // 0: none
  bool bad;
};

__device__ __forceinline__ Settings draw_settings(const DrawArgs& a, int row) {
  Settings s;
  float t = a.temperature ? a.temperature[row] : 1.0f;
  s.k = a.top_k ? max(a.top_k[row], 0) : 0;
  s.p = a.top_p ? a.top_p[row] : 1.0f;
  s.min_p = a.min_p ? a.min_p[row] : 0.0f;
  s.bad = !(t >= 0.0f && t <= FLT_MAX) || s.p != s.p || s.min_p != s.min_p;
  if (!(s.p < 1.0f)) s.p = 1.0f;
  if (!(s.min_p > 0.0f)) s.min_p = 0.0f;
  if (!(t > 0.0f && t <= FLT_MAX)) {                     // the best token alone
    t = 1.0f;
    s.k = 1;
    s.p = 1.0f;
    s.min_p = 0.0f;
  }
  if (s.min_p > 1.0f) s.k = 1;                           // no weight reaches it: the first one is kept
  s.inv_t = 1.0 / (double)t;
  s.grid = fminf(4.0f / t, FLT_MAX);
  return s;
}

__device__ __forceinline__ float draw_clean(float x) { return x == x ? fminf(x + 0.0f, FLT_MAX) : -INFINITY; }
__device__ __forceinline__ int draw_bin(float x, float grid) {
  return (int)fminf(fmaxf(floorf(x * grid), -1e9f), 1e9f);
}
__device__ __forceinline__ double draw_weight(float x, float top, double inv_t) {
  return x > -INFINITY ? exp(((double)x - (double)top) * inv_t) : 0.0;
}
// w in [0, 1] in units of 1 / unit (a power of two up to 2^51), rounded to nearest.
__device__ __forceinline__ unsigned long long draw_fix(double w, double unit) {
  return (unsigned long long)__double_as_longlong(fma(w, unit, 0x1p52)) & ((1ull << 52) - 1);
}
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

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_top(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
// Inclusive prefix sums over the wave's lanes.
template <typename T>
__device__ __forceinline__ T wave_scan(T v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

// A slice's logits, 4 * E of a thread: x[4 i + j] at t0 + 1024 i + 4 tid + j; -inf behind the row's end.
template <int E>
__device__ __forceinline__ void draw_load(const float* row, int t0, int V, int tid, float x[4 * E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int t = t0 + 1024 * i + 4 * tid;
    if (t + 3 < V) {
      const Four f = *(const Four*)(row + t);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = draw_clean(f.v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = t + j < V ? draw_clean(row[t + j]) : -INFINITY;
    }
  }
}

template <int E, bool LIMITS>
__global__ void __launch_bounds__(256) k_draw_scan(DrawArgs a) {
  __shared__ unsigned long long mass[kBins], sums[4];
  __shared__ uint32_t count[kBins];
  __shared__ float tops[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, slice = blockIdx.x, V = a.vocab;
  const Settings s = draw_settings(a, row);
  float x[4 * E];
  draw_load<E>(a.logits + (int64_t)row * V, slice * 1024 * E, V, tid, x);
  if (LIMITS && tid < kBins) {
    mass[tid] = 0;
    count[tid] = 0;
  }
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4 * E; ++i) top = fmaxf(top, x[i]);
  top = wave_top(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const int best = draw_bin(top, s.grid);
  unsigned long long sum = 0;
#pragma unroll
  for (int i = 0; i < 4 * E; ++i) {
    const unsigned long long w = draw_fix(draw_weight(x[i], top, s.inv_t), kSliceUnit);
    sum += w;
    if (LIMITS && x[i] > -INFINITY) {
      const int j = min(best - draw_bin(x[i], s.grid), kBins - 1);
      atomicAdd(&mass[j], w);
      atomicAdd(&count[j], 1u);
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  const int64_t at = (int64_t)row * a.slices + slice;
  if (tid == 0) {
    a.stat[at] = SliceStat{top, best, sums[0] + sums[1] + sums[2] + sums[3]};
    if (LIMITS && slice == 0) a.listed[row] = 0;
  }
  if (LIMITS && tid < kBins) {
    a.mass[at * kBins + tid] = mass[tid];
    a.count[at * kBins + tid] = count[tid];
  }
}

template <int E>
__global__ void __launch_bounds__(256) k_draw_list(DrawArgs a) {
  __shared__ double mass[kBins], half_mass[kBins], low_mass[4];
  __shared__ int count[kBins], half_count[kBins], low_count[4];
  __shared__ float tops[4];
  __shared__ RowPlan plan;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, slice = blockIdx.x, V = a.vocab;
  const Settings s = draw_settings(a, row);
  const SliceStat* stat = a.stat + (int64_t)row * a.slices;
  float top = -INFINITY;
  for (int i = tid; i < a.slices; i += 256) top = fmaxf(top, stat[i].top);
  top = wave_top(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const int bin = draw_bin(top, s.grid);
  // The row's bins: thread j of either half of the work group takes bin j of every other slice; bins that are the
  // row's last one or lower together (a slice's own last bin always is)
  const int j = tid & (kBins - 1), half = tid >> 7;
  double m = 0.0, lm = 0.0;
  int c = 0, lc = 0;
  for (int i = half; i < a.slices; i += 2) {
    const SliceStat t = stat[i];
    if (!(t.top > -INFINITY)) continue;
    const double f = exp(((double)t.top - (double)top) * s.inv_t) * (1.0 / kSliceUnit);
    const int off = bin - t.bin;                         // 0 or more
    const int64_t at = ((int64_t)row * a.slices + i) * kBins;
    if (j >= off && j < kBins - 1) {
      m += f * (double)a.mass[at + j - off];
      c += (int)a.count[at + j - off];
    }
    if (off >= kBins - 1 || j >= kBins - 1 - off) {
      lm += f * (double)a.mass[at + j];
      lc += (int)a.count[at + j];
    }
  }
  if (half) {
    half_mass[j] = m;
    half_count[j] = c;
  }
  lm = wave_sum(lm);
  lc = wave_sum(lc);
  if (lane == 0) {
    low_mass[wave] = lm;
    low_count[wave] = lc;
  }
  __syncthreads();
  if (!half) {
    m += half_mass[j];
    c += half_count[j];
    if (j == kBins - 1) {
      m = (low_mass[0] + low_mass[1]) + (low_mass[2] + low_mass[3]);
      c = low_count[0] + low_count[1] + low_count[2] + low_count[3];
    }
    mass[j] = m;
    count[j] = c;
  }
  __syncthreads();
  if (wave == 0) {                                       // sums up to each bin
    const double m0 = mass[2 * lane], m1 = mass[2 * lane + 1];
    const int c0 = count[2 * lane], c1 = count[2 * lane + 1];
    const double ms = wave_scan(m0 + m1, lane);
    const int cs = wave_scan(c0 + c1, lane);
    mass[2 * lane] = ms - m1;
    mass[2 * lane + 1] = ms;
    count[2 * lane] = cs - c1;
    count[2 * lane + 1] = cs;
  }
  __syncthreads();
  if (tid == 0) {
    RowPlan p{top, -INFINITY, bin, kBins, kBins - 1, 0, 0, 0.0, mass[kBins - 1]};
    if (top > -INFINITY) {
      auto first_count = [&](int n) {
        int i = 0;
        while (i < kBins - 1 && count[i] < n) ++i;
        return i;
      };
      int b1 = kBins;                                    // where top_k's or min_p's border lies
      if (s.k > 0 && s.k < count[kBins - 1]) b1 = s.k == 1 ? 0 : first_count(s.k);
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
      p.limited = b1 < kBins;
      p.first = b1;
      p.last = min(b1, kBins - 1);
      if (s.p < 1.0f) {
        // weight of what top_k and min_p keep: at least that of the bins before the border
        const double least = b1 == kBins ? mass[kBins - 1] : b1 > 0 ? mass[b1 - 1] : 0.0;
        int i = 0;
        while (i < min(b1, kBins - 1) && mass[i] < (double)s.p * least) ++i;
        p.first = i;
        p.last = b1 < kBins ? b1 : i;
      } else if (b1 == kBins) {
        p.last = -1;                                     // nothing to list
      }
      if (p.first > 0) {
        p.count0 = count[p.first < kBins ? p.first - 1 : kBins - 1];
        p.mass0 = mass[p.first < kBins ? p.first - 1 : kBins - 1];
      }
    } else {
      p.last = -1;
    }
    plan = p;
    if (slice == 0) a.plan[row] = p;
  }
  __syncthreads();
  const int first = plan.first, last = plan.last;
  if (first > last) return;
  const SliceStat own = stat[slice];
  if (!(own.top > -INFINITY) || min(bin - own.bin, kBins - 1) > last) return;
  float x[4 * E];
  const int t0 = slice * 1024 * E;
  draw_load<E>(a.logits + (int64_t)row * V, t0, V, tid, x);
#pragma unroll
  for (int i = 0; i < 4 * E; ++i) {
    const int at = x[i] > -INFINITY ? min(bin - draw_bin(x[i], s.grid), kBins - 1) : kBins;
    const bool in = at >= first && at <= last;
    const unsigned long long who = __ballot(in);
    if (!who) continue;
    int base = 0;
    if (lane == 0) base = atomicAdd(&a.listed[row], __popcll(who));
    base = __shfl(base, 0, 64) + __popcll(who & ((1ull << lane) - 1));
    if (in && base < kList)
      a.list[(int64_t)row * kList + base] = draw_key(x[i], t0 + 1024 * (i / 4) + 4 * tid + i % 4);
  }
}

// sums over the work group's threads up to and including this one's, in the order of threads
template <typename T>
__device__ __forceinline__ T group_scan(T v, T* parts, int tid, T& total) {
  const int lane = tid & 63, wave = tid >> 6;
  v = wave_scan(v, lane);
  __syncthreads();
  if (lane == 63) parts[wave] = v;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPickThreads / 64; ++w) {
    if (w < wave) before += parts[w];
    total += parts[w];
  }
  return v + before;
}

template <bool LIMITS>
__global__ void __launch_bounds__(kPickThreads) k_draw_pick(DrawArgs a, int slice_len, int unit_bits) {
  constexpr int kParts = 1024, NT = kPickThreads, NW = NT / 64;
  __shared__ unsigned long long list[LIMITS ? kList : 1], pm[LIMITS ? kParts : 1];
  __shared__ uint32_t pc[LIMITS ? kParts : 1];
  __shared__ unsigned long long ull[NW];
  __shared__ int ints[NW];
  __shared__ double dbl[NW];
  __shared__ float tops[NW];
  __shared__ int chosen, part, last_kept;
  __shared__ double share, before_slice;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x, V = a.vocab;
  const float* x = a.logits + (int64_t)row * V;
  const Settings s = draw_settings(a, row);
  const SliceStat* stat = a.stat + (int64_t)row * a.slices;
  const double unit = (double)(1ull << unit_bits);
  float u = a.uniforms[row];
  const bool bad = s.bad || !(u >= 0.0f && u < 1.0f);
  u = u >= 1.0f ? 1.0f - 0x1p-24f : u > 0.0f ? u : 0.0f;
  if (bad && tid == 0) atomicOr(a.err, kErrSample);
  RowPlan p{};
  if (LIMITS) {
    p = a.plan[row];
  } else {
    float top = -INFINITY;
    for (int i = tid; i < a.slices; i += NT) top = fmaxf(top, stat[i].top);
    top = wave_top(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, tops[w]);
    p.top = top;
    p.first = kBins;
    p.last = -1;
  }
  if (!(p.top > -INFINITY)) {                            // nothing to draw
    if (tid == 0) {
      a.tokens[row] = -1;
      if (a.logprobs) a.logprobs[row] = -INFINITY;
    }
    return;
  }
  auto bin_of = [&](float v) __attribute__((always_inline)) { return min(p.bin - draw_bin(v, s.grid), kBins - 1); };
  auto fixed = [&](float v) __attribute__((always_inline)) { return draw_fix(draw_weight(v, p.top, s.inv_t), unit); };

  unsigned long long border = 0;                         // listed keys from here on are kept
  int n_list = 0;
  bool in_list = true;
  // all that was listed: f(key); of the row itself where the list did not hold it
  auto candidates = [&](auto f) __attribute__((always_inline)) {
    if (in_list) {
      for (int i = tid; i < n_list; i += NT) f(list[i]);
    } else {
      for (int t = tid; t < V; t += NT) {
        const float v = draw_clean(x[t]);
        if (!(v > -INFINITY)) continue;
        const int b = bin_of(v);
        if (b >= p.first && b <= p.last) f(draw_key(v, t));
      }
    }
  };
  if constexpr (LIMITS) {
    if (p.first <= p.last) {
      n_list = a.listed[row];
      in_list = n_list <= kList;
      if (in_list)
        for (int i = tid; i < n_list; i += NT) list[i] = a.list[(int64_t)row * kList + i];
      __syncthreads();
      // The border: of the keys from `least` on in falling order, the one at which the count from count0 on reaches
      // want, or (want 0) the weight from mass0 on reaches goal.
      auto find = [&](unsigned long long least, int want, double goal) {
        unsigned long long lo = ~0ull, hi = 0;
        candidates([&](unsigned long long k) {
          if (k >= least) {
            lo = min(lo, k);
            hi = max(hi, k);
          }
        });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          lo = min(lo, __shfl_xor(lo, o, 64));
          hi = max(hi, __shfl_xor(hi, o, 64));
        }
        __syncthreads();
        if (lane == 0) ull[wave] = lo;
        __syncthreads();
        for (int w = 0; w < NW; ++w) lo = min(lo, ull[w]);
        __syncthreads();
        if (lane == 0) ull[wave] = hi;
        __syncthreads();
        for (int w = 0; w < NW; ++w) hi = max(hi, ull[w]);
        if (lo > hi) return least;                       // there are none
        int have = p.count0;
        unsigned long long held = (unsigned long long)(p.mass0 * unit);
        while (lo < hi) {
          const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 10);
          for (int i = tid; i < kParts; i += NT) {
            pm[i] = 0;
            pc[i] = 0;
          }
          __syncthreads();
          candidates([&](unsigned long long k) {
            if (k < lo || k > hi) return;
            const int i = kParts - 1 - (int)((k - lo) >> shift);       // falling
            atomicAdd(&pm[i], fixed(unordered((uint32_t)(k >> 32))));
            atomicAdd(&pc[i], 1u);
          });
          __syncthreads();
          const unsigned long long m0 = pm[2 * tid], m1 = pm[2 * tid + 1];
          const int c0 = (int)pc[2 * tid], c1 = (int)pc[2 * tid + 1];
          unsigned long long mt;
          int ct;
          const unsigned long long me = group_scan(m0 + m1, ull, tid, mt) - m1;
          const int ce = group_scan(c0 + c1, ints, tid, ct) - c1;
          if (tid == 0) part = INT32_MAX;
          __syncthreads();
          auto there = [&](int c, unsigned long long m) {
            return want > 0 ? have + c >= want : (double)(held + m) >= goal;
          };
          if (c0 && there(ce, me)) atomicMin(&part, 2 * tid);
          else if (c1 && there(ce + c1, me + m1)) atomicMin(&part, 2 * tid + 1);
          __syncthreads();
          const int at = part;
          if (at == INT32_MAX) return lo;                // not reached: all of them
          // what lies before that part
          if (at / 2 == tid) {
            ints[0] = at % 2 ? ce : ce - c0;
            ull[0] = at % 2 ? me : me - m0;
          }
          __syncthreads();
          have += ints[0];
          held += ull[0];
          const unsigned long long from = lo + ((unsigned long long)(kParts - 1 - at) << shift);
          const unsigned long long to = from + ((1ull << shift) - 1);
          lo = max(lo, from);
          hi = min(hi, to);
          __syncthreads();
          if (shift == 0) break;
        }
        return lo;
      };
      unsigned long long least = 0;
      if (p.limited && p.xm > -INFINITY) least = (unsigned long long)ordered(p.xm) << 32;
      if (p.limited && s.k > 0) least = max(least, find(least, s.k, 0.0));
      if (s.p < 1.0f) {
        unsigned long long sum = 0;
        candidates([&](unsigned long long k) {
          if (k >= least) sum += fixed(unordered((uint32_t)(k >> 32)));
        });
        unsigned long long all;
        if (!p.limited) {
          border = find(least, 0, (double)s.p * p.total * unit);     // no limit before it
        } else {
          group_scan(sum, ull, tid, all);
          border = find(least, 0, (double)s.p * ((double)all + p.mass0 * unit));
        }
      } else {
        border = least;
      }
    }
  }
  // Weights kept in each slice, and which slice the token falls into.  The slices' sums are formed by one wave
  // each, in turn; thread 0 adds them up in their order, so they are kept where the list was.
  auto kept = [&](float v, int t) __attribute__((always_inline)) {
    if (!LIMITS) return v > -INFINITY;
    if (!(v > -INFINITY)) return false;
    const int b = bin_of(v);
    return b < p.first || (b <= p.last && draw_key(v, t) >= border);
  };
  // one slice after the other, the listed ones' share by going through them
  __shared__ unsigned long long add[NW];
  double sum = 0.0;                                      // of all slices, in every thread
  // pass 0 sums up, pass 1 finds the slice
  if (tid == 0) {
    chosen = -1;
    last_kept = -1;
  }
  __syncthreads();
  double target = 0.0;
  for (int pass = 0; pass < 2; ++pass) {
    double run = 0.0;
    for (int s0 = 0; s0 < a.slices; s0 += NW) {
      const int i = s0 + wave;
      double part_sum = 0.0;
      if (i < a.slices && stat[i].top > -INFINITY) {
        const SliceStat t = stat[i];
        const double f = exp(((double)t.top - (double)p.top) * s.inv_t);
        if (!LIMITS || p.first >= kBins) {
          part_sum = f * ((double)t.sum * (1.0 / kSliceUnit));
        } else {
          const int off = p.bin - t.bin;
          unsigned long long m = 0;
          const int64_t at = ((int64_t)row * a.slices + i) * kBins;
          for (int b = lane; b < kBins - 1; b += 64)
            if ((int64_t)off + b < p.first) m += a.mass[at + b];
          m = wave_sum(m);
          unsigned long long l = 0;
          if (p.first <= p.last) {
            const int from = i * slice_len, to = min(V, from + slice_len);
            if (in_list) {
              for (int q = lane; q < n_list; q += 64) {
                const unsigned long long k = list[q];
                const int at_t = (int)(0xFFFFFFFFu - (uint32_t)k);
                if (k >= border && at_t >= from && at_t < to) l += fixed(unordered((uint32_t)(k >> 32)));
              }
            } else {
              for (int q = from + lane; q < to; q += 64) {
                const float v = draw_clean(x[q]);
                if (!(v > -INFINITY)) continue;
                const int b = bin_of(v);
                if (b >= p.first && b <= p.last && draw_key(v, q) >= border) l += fixed(v);
              }
            }
            l = wave_sum(l);
          }
          part_sum = f * ((double)m * (1.0 / kSliceUnit)) + (double)l / unit;
        }
      }
      __syncthreads();
      if (lane == 0) dbl[wave] = part_sum;
      __syncthreads();
      for (int w = 0; w < NW; ++w) {
        const double next = run + dbl[w];
        if (pass == 1 && tid == 0 && dbl[w] > 0.0) {
          if (last_kept < 0 || !(share > target)) {      // not found yet: this one, or a later one
            last_kept = s0 + w;
            before_slice = run;
            share = next;
          }
        }
        run = next;
      }
      __syncthreads();
    }
    if (pass == 0) {
      sum = run;
      target = (double)u * sum;
    }
  }
  __syncthreads();
  // the token in that slice
  const int s_at = max(last_kept, 0);
  const double want = target - before_slice;
  double run = 0.0;
  const int from = s_at * slice_len, to = min(V, from + slice_len);
  if (tid == 0) chosen = -1;
  __syncthreads();
  for (int t0 = from; t0 < to; t0 += 4 * NT) {
    const int t = t0 + 4 * tid;
    double w[4], mine = 0.0;
    int lastk = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = t + j < to ? draw_clean(x[t + j]) : -INFINITY;
      w[j] = kept(v, t + j) ? draw_weight(v, p.top, s.inv_t) : 0.0;
      mine += w[j];
      if (w[j] > 0.0) lastk = t + j;
    }
    double total;
    const double upto = group_scan(mine, dbl, tid, total);
    if (tid == 0) part = INT32_MAX;
    __syncthreads();
    double c = run + (upto - mine);
    int hit = INT32_MAX;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c += w[j];
      if (w[j] > 0.0 && c > want && hit == INT32_MAX) hit = t + j;
    }
    if (hit != INT32_MAX) atomicMin(&part, hit);
    if (lastk >= 0) atomicMax(&chosen, lastk);           // where rounding leaves none: the last one
    __syncthreads();
    if (part != INT32_MAX) break;
    run += total;
    __syncthreads();
  }
  if (tid == 0) {
    const int t = part != INT32_MAX ? part : max(chosen, from);
    a.tokens[row] = t;
    if (a.logprobs) a.logprobs[row] = (float)(((double)draw_clean(x[t]) - (double)p.top) * s.inv_t - log(sum));
  }
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
  RuleArgs a{logits, out, vocab, rows, r, c->d_err};
  if (a.r.hist_len == 0) a.r.history = nullptr;
  hipLaunchKernelGGL(k_adjust, dim3((unsigned)((vocab + kRuleSlice - 1) / kRuleSlice), (unsigned)rows), dim3(256), 0,
                     c->stream, a);
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
  const int long_slices = (vocab + 8191) / 8192;
  const bool large = most * long_slices >= 2 * (int64_t)c->n_cu || long_slices > 64;
  const int slice = large ? 8192 : 2048, slices = (vocab + slice - 1) / slice;
  // temperatures, read on the device, may ask for the best token: limits too
  const bool limits = temperature || top_k || top_p || min_p;
  const int64_t per_row = (int64_t)slices * sizeof(SliceStat) +
                          (limits ? (int64_t)slices * kBins * 12 + sizeof(RowPlan) + 8 + (int64_t)kList * 8 : 0);
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
    a.plan = (RowPlan*)take(most * sizeof(RowPlan));
    a.listed = (int32_t*)take(most * 8);
    a.count = (uint32_t*)take(most * slices * kBins * 4);
  }
  int bits = 1;                                          // of a sum of vocab weights, and one more
  while ((1 << bits) < vocab) ++bits;
  const int unit = std::min(51, 62 - bits);
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
#define TMZ_DRAW(E)                                                                        \
  if (limits) {                                                                            \
    hipLaunchKernelGGL((k_draw_scan<E, true>), grid, dim3(256), 0, c->stream, a);          \
    hipLaunchKernelGGL((k_draw_list<E>), grid, dim3(256), 0, c->stream, a);                \
  } else {                                                                                 \
    hipLaunchKernelGGL((k_draw_scan<E, false>), grid, dim3(256), 0, c->stream, a);         \
  }
    if (large) {
      TMZ_DRAW(8)
    } else {
      TMZ_DRAW(2)
    }
#undef TMZ_DRAW
    if (limits)
      hipLaunchKernelGGL((k_draw_pick<true>), dim3((unsigned)n), dim3(kPickThreads), 0, c->stream, a, slice, unit);
    else
      hipLaunchKernelGGL((k_draw_pick<false>), dim3((unsigned)n), dim3(kPickThreads), 0, c->stream, a, slice, unit);
  }
  return hip_status(c, hipGetLastError(), "sample");
}

}  // extern "C"
