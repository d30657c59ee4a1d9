// Choosing the next tokens: the logits of a few rows of hidden states over the embedding, and beam
// search's selection among them.
#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "tmz_device.h"
#include "tmz_internal.h"

namespace tmz {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Logits of few rows: out[m][t] = x[m] . E[t].  Bound by the bytes of E (2 M flops a byte of bf16), so E
// is read once for up to 64 rows, straight into matrix operands: lane l of a wave loads 16 bytes of
// vocabulary row l % 16 at byte 16 (l / 16) of a 64-byte step, the same piece of hidden state l % 16 is the
// other operand (from the caches: all of x is small), and no LDS or barrier stands in the loop.  bf16: a
// 16x16x32 instruction a step; fp32: four 16x16x4, the lane's k-th value in the k-th.  The four waves of a
// work group share VT x 16 vocabulary rows and divide the steps, so that few rows of a small vocabulary fill the
// device too; their sums are joined in LDS in a fixed order.
// grid: tiles of hidden states x vocabulary tiles (the former fastest: they meet in the caches).
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ v4f logits_step(uint4 a, uint4 b, v4f c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b),
                                                   c, 0, 0, 0);
  } else {
    const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
}

template <typename T, int MT, int VT>
__global__ void __launch_bounds__(256) k_logits(const T* __restrict__ x, const T* __restrict__ E, int64_t M,
                                                int64_t d, int64_t V, float* __restrict__ out,
                                                int mtiles) {
  __shared__ v4f red[3][MT * VT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m0 = (int64_t)(blockIdx.x % mtiles) * 16 * MT, t0 = (int64_t)(blockIdx.x / mtiles) * 16 * VT;
  const int64_t bytes = d * (int64_t)sizeof(T);
  const int whole = (int)(bytes / 64);                   // steps
  // rows past the end are read as the last one and not stored
  const char *xp[MT], *ep[VT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + 16 * i + (lane & 15);
    xp[i] = (const char*)(x + (m < M ? m : M - 1) * d) + (lane >> 4) * 16;
  }
#pragma unroll
  for (int i = 0; i < VT; ++i) {
    const int64_t t = t0 + 16 * i + (lane & 15);
    ep[i] = (const char*)(E + (t < V ? t : V - 1) * d) + (lane >> 4) * 16;
  }
  v4f acc[MT][VT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < VT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  // GS steps at a time, the waves in turn: all their loads first, a row's pieces next to each other
  constexpr int GS = MT * VT >= 16 ? 2 : 4;
  auto take = [&](int s, auto count) __attribute__((always_inline)) {
    constexpr int C = decltype(count)::value;
    uint4 a[VT][C], b[MT][C];
#pragma unroll
    for (int j = 0; j < VT; ++j)
#pragma unroll
      for (int u = 0; u < C; ++u) a[j][u] = *(const uint4*)(ep[j] + (int64_t)(s + u) * 64);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int u = 0; u < C; ++u) b[i][u] = *(const uint4*)(xp[i] + (int64_t)(s + u) * 64);
#pragma unroll
    for (int u = 0; u < C; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < VT; ++j) acc[i][j] = logits_step<T>(a[j][u], b[i][u], acc[i][j]);
  };
  int s = wave * GS;
  for (; s + GS <= whole; s += 4 * GS) take(s, std::integral_constant<int, GS>());
  for (; s < whole; ++s) take(s, std::integral_constant<int, 1>());
  if (wave == 0 && whole * 64 < bytes) {                 // the last step is half a one
    const bool in = (lane >> 4) * 16 < bytes - (int64_t)whole * 64;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    uint4 a[VT], b[MT];
#pragma unroll
    for (int j = 0; j < VT; ++j) a[j] = in ? *(const uint4*)(ep[j] + (int64_t)whole * 64) : zero;
#pragma unroll
    for (int i = 0; i < MT; ++i) b[i] = in ? *(const uint4*)(xp[i] + (int64_t)whole * 64) : zero;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < VT; ++j) acc[i][j] = logits_step<T>(a[j], b[i], acc[i][j]);
  }
  if (wave > 0)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < VT; ++j) red[wave - 1][i * VT + j][lane] = acc[i][j];
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < VT; ++j) {
#pragma unroll
      for (int w = 0; w < 3; ++w) acc[i][j] += red[w][i * VT + j][lane];
      const int64_t m = m0 + 16 * i + (lane & 15), t = t0 + 16 * j + (lane >> 4) * 4;
      if (m >= M) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (t + r < V) out[m * V + t + r] = acc[i][j][r];
    }
}

// The same with all of x in LDS: work groups, as many as LDS lets run, walk the vocabulary, a wave 16 rows of E at
// a time, GS steps ahead of the matrix instructions.  E's bytes are then all that passes the caches
// (one row of 128256 x 2560 139 -> 110 us, 5.9 TB/s; 16 rows 156 -> 131, 32 rows 166 -> 137).  16 rows' reads fall
// on all banks: rows are 16 bytes apart beyond their length, or (DENSE, whole 128 bytes) piece c of 16 bytes of row m
// lies at c ^ (m % 8).
template <typename T, int MT, int KB, int NW, int GS, bool DENSE>
__global__ void __launch_bounds__(64 * NW) k_logits_walk(const T* __restrict__ x, const T* __restrict__ E,
                                                     int M, int d, int64_t V, float* __restrict__ out) {
  __shared__ __align__(16) char xs[KB * 1024];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bytes = d * (int)sizeof(T), pitch = DENSE ? bytes : bytes + 16, row16 = bytes / 16;
  constexpr int turn = DENSE ? 7 : 0;
  for (int i = threadIdx.x; i < M * row16; i += 64 * NW) {
    const int m = i / row16, c = i - m * row16;
    *(uint4*)(xs + m * pitch + (c ^ (m & turn)) * 16) = ((const uint4*)x)[i];
  }
  __syncthreads();
  const int whole = bytes / 64;
  const int g16 = (lane >> 4) * 16;
  int xo[MT], xm[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = 16 * i + (lane & 15) < M ? 16 * i + (lane & 15) : M - 1;
    xo[i] = m * pitch;
    xm[i] = (m & turn) * 16;
  }
  const int64_t tiles = (V + 15) / 16;
  for (int64_t tile = (int64_t)blockIdx.x * NW + wave; tile < tiles; tile += (int64_t)gridDim.x * NW) {
    const int64_t t = tile * 16 + (lane & 15);
    const char* ep = (const char*)(E + (t < V ? t : V - 1) * d) + g16;
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    auto use = [&](uint4 a, int s) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[i] = logits_step<T>(a, *(const uint4*)(xs + xo[i] + ((s * 64 + g16) ^ xm[i])), acc[i]);
    };
    uint4 a[2][GS];
    int s = 0;
    if (GS <= whole)
#pragma unroll
      for (int u = 0; u < GS; ++u) a[0][u] = *(const uint4*)(ep + u * 64);
    // two groups in turn, so that registers need no index
    for (; s + 2 * GS <= whole; s += 2 * GS) {
#pragma unroll
      for (int u = 0; u < GS; ++u) a[1][u] = *(const uint4*)(ep + (s + GS + u) * 64);
#pragma unroll
      for (int u = 0; u < GS; ++u) use(a[0][u], s + u);
      if (s + 3 * GS <= whole)
#pragma unroll
        for (int u = 0; u < GS; ++u) a[0][u] = *(const uint4*)(ep + (s + 2 * GS + u) * 64);
#pragma unroll
      for (int u = 0; u < GS; ++u) use(a[1][u], s + GS + u);
    }
    if (s + GS <= whole) {
#pragma unroll
      for (int u = 0; u < GS; ++u) use(a[0][u], s + u);
      s += GS;
    }
    for (; s < whole; ++s) use(*(const uint4*)(ep + s * 64), s);
    if (whole * 64 < bytes) {                            // half a step
      const bool in = g16 < bytes - whole * 64;
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
      const uint4 e = in ? *(const uint4*)(ep + whole * 64) : zero;
#pragma unroll
      for (int i = 0; i < MT; ++i)
        acc[i] = logits_step<T>(e, in ? *(const uint4*)(xs + xo[i] + ((whole * 64 + g16) ^ xm[i])) : zero, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = 16 * i + (lane & 15);
      const int64_t t4 = tile * 16 + (lane >> 4) * 4;
      if (m < M)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t4 + r < V) out[m * V + t4 + r] = acc[i][r];
    }
  }
}

template <typename T, int MT>
static void logits_as(const T* x, const T* E, int64_t M, int64_t d, int64_t V, float* out, int n_cu,
                      hipStream_t s) {
  // x in LDS where the vocabulary gives every compute unit four tiles of 16 rows (M = 3, d = 2560 in bf16: 16500 rows
  // 24 against 33 us of k_logits, 16000 rows 23 against 17, 1000 rows 20 against 6): two work groups of eight waves
  // on a compute unit while x takes half of LDS, else one, of sixteen waves where eight have more than a tile each
  // (M = 32, d = 1536: 33000 rows 38 -> 34 us; 32003 rows 24 with eight, 33 with sixteen).
  const int64_t bytes = d * (int64_t)sizeof(T), tiles = (V + 15) / 16, lds = M * (bytes + 16);
  const unsigned two = (unsigned)std::min<int64_t>((tiles + 7) / 8, 2 * n_cu);
  const unsigned one = (unsigned)std::min<int64_t>((tiles + 15) / 16, n_cu);
#define TMZ_WALK(MTV, KB, NW, GS, DENSE, GRID)                                                              \
  hipLaunchKernelGGL((k_logits_walk<T, MTV, KB, NW, GS, DENSE>), dim3(GRID), dim3(64 * NW), 0, s, x, E, (int)M, \
                     (int)d, V, out)
  if (M <= 16 * MT && tiles >= 4 * (int64_t)n_cu) {
    const bool dense = bytes % 128 == 0 && M * bytes <= 160 * 1024;
    const unsigned half = std::min(two, (unsigned)n_cu);
    constexpr int GS = MT == 8 ? 4 : 8;
    if constexpr (MT == 1) {
      if (lds <= 80 * 1024) {
        TMZ_WALK(1, 80, 8, 8, false, two);
        return;
      }
    }
    if constexpr (MT <= 4) {
      if (dense && tiles > 8 * (int64_t)n_cu) {
        TMZ_WALK(MT, 160, 16, 4, true, one);
        return;
      }
    }
    if (lds <= 160 * 1024) {
      TMZ_WALK(MT, 160, 8, GS, false, half);
      return;
    }
    if constexpr (MT <= 4) {
      if (dense) {
        TMZ_WALK(MT, 160, 8, GS, true, half);
        return;
      }
    }
  }
#undef TMZ_WALK
  if constexpr (MT <= 4) {
    const int mt = (int)((M + 16 * MT - 1) / (16 * MT));
    // 64 vocabulary rows a work group where that still makes one for every compute unit (M = 32, 32003 x 1536:
    // 501 work groups of 64 rows 24 us, 2001 of 16 rows 36)
    if ((V + 63) / 64 * mt >= n_cu)
      hipLaunchKernelGGL((k_logits<T, MT, 4>), dim3((unsigned)((V + 63) / 64 * mt)), dim3(256), 0, s, x, E, M, d,
                         V, out, mt);
    else
      hipLaunchKernelGGL((k_logits<T, MT, 1>), dim3((unsigned)((V + 15) / 16 * mt)), dim3(256), 0, s, x, E, M, d,
                         V, out, mt);
  }
}

hipError_t launch_logits(const void* x, const void* E, termezo_dtype dt, int64_t M, int64_t d,
                         int64_t V, float* out, int n_cu, hipStream_t s) {
  const int64_t tiles = (V + 15) / 16, bytes = M * d * (dt == TERMEZO_BF16 ? 2 : 4);
  // rows of x a work group takes: fewer where that still makes no more than one for every compute unit (64 rows,
  // d = 2560 in bf16, 1000 vocabulary rows: 64 at a time 14.8 us, 32 9.7, 16 7.6; 4000: 18.1, 18.1, 21.3)
  int mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  while (mt > 1 && tiles * ((M + 8 * mt - 1) / (8 * mt)) <= n_cu) mt /= 2;
  // all of them, up to 128, if they fit LDS (70 rows of 512 in bf16, 32000 vocabulary rows: 25 -> 16 us; 128: 27 -> 22)
  if (M > 64 && M <= 128 && bytes + 16 * M <= 160 * 1024 && tiles >= 4 * (int64_t)n_cu) mt = 8;
#define TMZ_LOGITS(T)                                                                     \
  if (mt == 1) logits_as<T, 1>((const T*)x, (const T*)E, M, d, V, out, n_cu, s);          \
  else if (mt == 2) logits_as<T, 2>((const T*)x, (const T*)E, M, d, V, out, n_cu, s);     \
  else if (mt == 4) logits_as<T, 4>((const T*)x, (const T*)E, M, d, V, out, n_cu, s);     \
  else logits_as<T, 8>((const T*)x, (const T*)E, M, d, V, out, n_cu, s)
  if (dt == TERMEZO_BF16) {
    TMZ_LOGITS(uint16_t);
  } else {
    TMZ_LOGITS(float);
  }
#undef TMZ_LOGITS
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Beam selection in two launches.
//
// k_beam_scan reads the logits once, a wave 1024 of them in registers, and leaves per wave the largest and
// the sum of exp(x - largest), and the largest of every segment (16, 64, 256 or 1024 logits).
// k_beam_pick, a work group per search, forms the beams' log-sum-exps (fp64) and the segments' best scores
// (score + x) - lse (fp64).  A lower bound of the n_out-th best score is the n_out-th largest of the
// maxima of 64 disjoint sets of segments: no continuation below it can be chosen, and only segments that
// reach it are looked at again.  The few continuations found are ranked by counting; where they are many
// (many equal logits) they are taken in rounds, best first.  Continuations of score -inf fill what is left,
// lowest index first.  The scan is bound by the bytes of the logits, the pick by its chain of reads.
// ---------------------------------------------------------------------------
struct BeamArgs {
  const float *logits, *scores;
  const uint8_t* finished;
  int32_t beams, vocab, n_out, eos;
  float* out_scores;
  int32_t *out_tokens, *out_parents;
  uint8_t* out_finished;
  const int32_t* history;
  int32_t* out_history;
  int64_t hist_len;
  // scratch: [row][waves] (largest, sum), [row][segs]
  float2* part;
  float* seg;
  int32_t waves, segs, seg_shift;
};

constexpr int kScan = 1024;           // logits a wave

struct __attribute__((packed, aligned(4))) Float4 {
  float v[4];
};

// NaN counts as -inf, -0 as 0.
__device__ __forceinline__ float clean_logit(float x) { return x == x ? x + 0.0f : -INFINITY; }

// v of the lane that a data-parallel move names (quad permutation, rotation of 16 lanes).
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, false));
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kTurn4 = 0x124, kTurn8 = 0x128;

template <int SHIFT>
__global__ void __launch_bounds__(256) k_beam_scan(BeamArgs a) {
  const int lane = threadIdx.x & 63, w = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t row = blockIdx.y;
  if (w >= a.waves || (a.finished && a.finished[row])) return;   // whole wave
  const float* x = a.logits + row * a.vocab;
  const int t0 = w * kScan + lane * 4;
  float v[4][4], b[4];
  if (w * kScan + kScan <= a.vocab) {                    // whole wave
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Float4 f = *(const Float4*)(x + t0 + i * 256);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = f.v[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = t0 + i * 256 + j;
        const float f = x[t < a.vocab ? t : a.vocab - 1];
        v[i][j] = t < a.vocab ? f : -INFINITY;
      }
  }
  float* seg = a.seg + row * a.segs;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = clean_logit(v[i][j]);
    b[i] = fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3]));
    b[i] = fmaxf(b[i], moved<kSwap1>(b[i]));
    b[i] = fmaxf(b[i], moved<kSwap2>(b[i]));
    const int t = t0 + i * 256;
    if (SHIFT == 4 && lane % 4 == 0 && t < a.vocab) seg[t >> 4] = b[i];
    b[i] = fmaxf(b[i], moved<kTurn4>(b[i]));
    b[i] = fmaxf(b[i], moved<kTurn8>(b[i]));
    if (SHIFT == 6 && lane % 16 == 0 && t < a.vocab) seg[t >> 6] = b[i];
    if (SHIFT == 8) {
      b[i] = fmaxf(b[i], __shfl_xor(b[i], 16, 64));
      b[i] = fmaxf(b[i], __shfl_xor(b[i], 32, 64));
      if (lane == 0 && t < a.vocab) seg[t >> 8] = b[i];
    }
  }
  float m = fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]));
  if (SHIFT != 8) {
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
  }
  if (SHIFT == 10 && lane == 0) seg[w] = m;
  const float ref = m == -INFINITY ? 0.0f : m;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      s[j] += __builtin_amdgcn_exp2f((v[i][j] - ref) * 1.4426950408889634f);
  float sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lane == 0) a.part[row * a.waves + w] = make_float2(m, sum);
}

constexpr int kPickWaves = 8, kPick = 64 * kPickWaves, kMaxList = 1024, kMaxCand = 512, kMaxOut = 64;

__device__ __forceinline__ bool before(double v, int i, double w, int j) {
  return v > w || (v == w && i < j);
}

__global__ void __launch_bounds__(kPick) k_beam_pick(BeamArgs a) {
  __shared__ double lse[64], own[64], cv[kMaxCand], rv[kPickWaves];
  __shared__ float lmax[kPickWaves][64], bound;
  __shared__ int list[kMaxList], ci[kMaxCand], ri[kPickWaves], n_list, n_cand, pick[kMaxOut], n_pick;
  __shared__ float pv[kMaxOut];
  __shared__ bool done[64];
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int W = a.beams, V = a.vocab, segs = a.segs, shift = a.seg_shift, eos = a.eos;
  const int64_t row0 = (int64_t)g * W;
  if (tid == 0) n_list = n_cand = 0;
  // The usual search's segments (eight beams, a segment a thread) stay in registers; their loads and
  // those of the parts go out together.
  const bool held = W <= 8 && segs <= kPick;
  float seg_max[8];
  if (held)
#pragma unroll
    for (int u = 0; u < 8; ++u)
      seg_max[u] = a.seg[(row0 + (u < W ? u : W - 1)) * segs + (tid < segs ? tid : segs - 1)];
  for (int b = wave; b < W; b += kPickWaves) {
    const bool fin = a.finished && a.finished[row0 + b];
    const float sc = a.scores[row0 + b];
    const float2* part = a.part + (row0 + b) * a.waves;
    const float2 none = make_float2(-INFINITY, 0.0f);
    const float2 p0 = lane < a.waves ? part[lane] : none, p1 = lane + 64 < a.waves ? part[lane + 64] : none;
    double l = INFINITY;                                 // no continuations
    if (!fin) {
      float m = fmaxf(p0.x, p1.x);
      for (int i = lane + 128; i < a.waves; i += 64) m = fmaxf(m, part[i].x);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
      double s = 0.0;
      auto add = [&](float2 p) __attribute__((always_inline)) {
        if (p.x > -INFINITY) s += (double)p.y * exp((double)p.x - (double)m);
      };
      add(p0);
      add(p1);
      for (int i = lane + 128; i < a.waves; i += 64) add(part[i]);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      l = (double)m + log(s);
      if (!(l > -INFINITY && l < INFINITY)) l = INFINITY;
    }
    if (lane == 0) {
      lse[b] = l;
      own[b] = sc == sc ? (double)sc : -INFINITY;
      done[b] = fin;
    }
  }
  __syncthreads();
  // score of a logit of beam b; x (clean) is not looked at where the beam is finished: eos has its score
  auto score = [&](int b, float x, bool is_eos) __attribute__((always_inline)) {
    const double v = lse[b] < INFINITY ? (own[b] + (double)x) - lse[b] : -INFINITY;
    if (done[b]) return is_eos ? own[b] : (double)-INFINITY;
    return v == v ? v : (double)-INFINITY;
  };
  // every segment's best, eight loads at a time: f(segment, score)
  auto segments = [&](auto f) __attribute__((always_inline)) {
    if (held) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (u < W && tid < segs) f(u * segs + tid, score(u, seg_max[u], eos >> shift == tid));
      return;
    }
    for (int j = tid; j < segs; j += kPick)
      for (int b0 = 0; b0 < W; b0 += 8) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = a.seg[(row0 + (b0 + u < W ? b0 + u : W - 1)) * segs + j];
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (b0 + u < W) f((b0 + u) * segs + j, score(b0 + u, x[u], eos >> shift == j));
      }
  };
  // all logits of listed segments, sixteen of a thread at a time: f(index, score)
  auto elements = [&](int n, bool all, auto f) __attribute__((always_inline)) {
    const int64_t total = (int64_t)n << shift;
    for (int64_t e0 = (int64_t)tid * 4; e0 < total; e0 += 4 * 4 * kPick) {
      float x[4][4];
      int bb[4], tt[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t e = e0 + u * 4 * kPick;
        const int at = e < total ? (int)(e >> shift) : n - 1, s = all ? at : list[at];
        bb[u] = s / segs;
        tt[u] = ((s - bb[u] * segs) << shift) + (int)(e & ((1 << shift) - 1));
        const float* row = a.logits + (row0 + bb[u]) * V;
        if (tt[u] + 3 < V) {
          const Float4 y = *(const Float4*)(row + tt[u]);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[u][j] = y.v[j];
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[u][j] = row[tt[u] + j < V ? tt[u] + j : V - 1];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (e0 + u * 4 * kPick < total && tt[u] + j < V)
            f(bb[u] * V + tt[u] + j, score(bb[u], clean_logit(x[u][j]), tt[u] + j == eos));
    }
  };
  // the bound in fp32, rounded down (a score between it and the exact one does no harm)
  double best = -INFINITY;
  segments([&](int, double v) { best = fmax(best, v); });
  lmax[wave][lane] = __double2float_rd(best);
  __syncthreads();
  if (wave == 0) {
    float m = lmax[0][lane];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w) m = fmaxf(m, lmax[w][lane]);
    int rank = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) {
      const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), i));
      rank += o > m || (o == m && i < lane);
    }
    if (rank == a.n_out - 1) bound = m;
  }
  __syncthreads();
  const double T = (double)bound;
  auto wanted = [&](double v) __attribute__((always_inline)) { return v >= T && v > -INFINITY; };
  segments([&](int s, double v) {
    if (wanted(v)) {
      const int i = atomicAdd(&n_list, 1);
      if (i < kMaxList) list[i] = s;
    }
  });
  __syncthreads();
  const bool all = n_list > kMaxList;                    // too many to list
  const int nl = all ? W * segs : n_list;
  if (!all)
    elements(nl, false, [&](int x, double v) {
      if (wanted(v)) {
        const int k = atomicAdd(&n_cand, 1);
        if (k < kMaxCand) {
          cv[k] = v;
          ci[k] = x;
        }
      }
    });
  __syncthreads();
  if (!all && n_cand <= kMaxCand) {
    const int nc = n_cand;
    for (int i = tid; i < nc; i += kPick) {
      const double v = cv[i];
      const int x = ci[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < nc; ++j) rank += before(cv[j], ci[j], v, x);
      if (rank < a.n_out) {
        pick[rank] = x;
        pv[rank] = (float)v;
      }
    }
    if (tid == 0) n_pick = nc < a.n_out ? nc : a.n_out;
    __syncthreads();
  } else {                                               // rounds: the best one behind the last
    double lv = INFINITY;
    int li = -1, r = 0;
    for (; r < a.n_out; ++r) {
      double bv = -INFINITY;
      int bi = INT32_MAX;
      elements(nl, all, [&](int x, double v) {
        if (wanted(v) && before(lv, li, v, x) && before(v, x, bv, bi)) {
          bv = v;
          bi = x;
        }
      });
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const double v = __shfl_xor(bv, o, 64);
        const int x = __shfl_xor(bi, o, 64);
        if (before(v, x, bv, bi)) {
          bv = v;
          bi = x;
        }
      }
      if (lane == 0) {
        rv[wave] = bv;
        ri[wave] = bi;
      }
      __syncthreads();
      for (int w = 0; w < kPickWaves; ++w)
        if (before(rv[w], ri[w], bv, bi)) {
          bv = rv[w];
          bi = ri[w];
        }
      __syncthreads();
      if (!(bv > -INFINITY)) break;                      // the same in every thread
      lv = bv;
      li = bi;
      if (tid == 0) {
        pick[r] = bi;
        pv[r] = (float)bv;
      }
    }
    if (tid == 0) n_pick = r;
    __syncthreads();
  }
  if (wave == 0 && n_pick < a.n_out) {                   // all finite ones are in: the first others
    int have = n_pick;
    for (int64_t x0 = 0; have < a.n_out && x0 < (int64_t)W * V; x0 += 64) {
      const int64_t x = x0 + lane;
      bool free = x < (int64_t)W * V;
      if (free) {
        const int b = (int)(x / V), t = (int)(x % V);
        free = !(score(b, clean_logit(a.logits[(row0 + b) * V + t]), t == eos) > -INFINITY);
      }
      const unsigned long long mask = __ballot(free);
      const int at = have + __popcll(mask & ((1ull << lane) - 1));
      if (free && at < a.n_out) {
        pick[at] = (int)x;
        pv[at] = -INFINITY;
      }
      have += __popcll(mask);
    }
  }
  __syncthreads();
  const int64_t o0 = (int64_t)g * a.n_out;
  for (int r = tid; r < a.n_out; r += kPick) {
    const int b = pick[r] / V, t = pick[r] % V;
    a.out_scores[o0 + r] = pv[r];
    a.out_tokens[o0 + r] = t;
    a.out_parents[o0 + r] = b;
    if (a.out_finished) a.out_finished[o0 + r] = done[b] || t == eos;
    if (a.out_history) a.out_history[(o0 + r) * (a.hist_len + 1) + a.hist_len] = t;
  }
  if (a.out_history) {                                   // eight loads of a thread at a time
    const int T = (int)a.hist_len, total = a.n_out * T;  // at most 64 x 2^24
    for (int i0 = tid; i0 < total; i0 += 8 * kPick) {
      int32_t x[8];
      int r[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + u * kPick < total ? i0 + u * kPick : total - 1;
        r[u] = i / T;
        x[u] = a.history[(row0 + pick[r[u]] / V) * T + (i - r[u] * T)];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + u * kPick;
        if (i < total) a.out_history[(o0 + r[u]) * (T + 1) + (i - r[u] * T)] = x[u];
      }
    }
  }
}

}  // namespace tmz

using namespace tmz;

namespace {

termezo_status gfail(termezo_ctx* c, const char* msg) {
  c->last_error = msg;
  return TERMEZO_ERR_INVALID_ARG;
}
termezo_status hip_status(termezo_ctx* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return TERMEZO_OK;
  (void)hipGetLastError();                               // reported here, not by the next launch
  c->last_error = std::string(what) + ": " + hipGetErrorString(e);
  return e == hipErrorOutOfMemory ? TERMEZO_ERR_OOM : TERMEZO_ERR_DEVICE;
}
bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace

extern "C" {

termezo_status termezo_logits(termezo_ctx* c, const void* x, const void* E, termezo_dtype dtype,
                              int64_t M, int64_t d, int64_t vocab, float* logits) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!x || !E || !logits || !aligned(x, 16) || !aligned(E, 16) || !aligned(logits, 16))
    return gfail(c, "logits: null or misaligned pointer");
  if ((dtype != TERMEZO_F32 && dtype != TERMEZO_BF16) || M <= 0 || M > 65535 || d <= 0 || d % 16 != 0 ||
      d > (1 << 24) || vocab <= 0 || vocab > (1 << 24))
    return gfail(c, "logits: a size or the type is out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "logits");
  return hip_status(c, launch_logits(x, E, dtype, M, d, vocab, logits, c->n_cu, c->stream), "logits");
}

termezo_status termezo_beam_select(termezo_ctx* c, const float* logits, const float* scores,
                                   const uint8_t* finished, int32_t groups, int32_t beams,
                                   int32_t vocab, int32_t n_out, int32_t eos, float* out_scores,
                                   int32_t* out_tokens, int32_t* out_parents,
                                   uint8_t* out_finished, const int32_t* history,
                                   int32_t* out_history, int64_t hist_len) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!logits || !scores || !out_scores || !out_tokens || !out_parents || (history && !out_history) ||
      (out_history && !history && hist_len != 0) ||
      !aligned(logits, 4) || !aligned(scores, 4) || !aligned(out_scores, 4) || !aligned(out_tokens, 4) ||
      !aligned(out_parents, 4) || !aligned(history, 4) || !aligned(out_history, 4))
    return gfail(c, "beam_select: null or misaligned pointer");
  if (groups <= 0 || groups > 65535 || beams <= 0 || beams > 64 || vocab <= 0 || vocab > (1 << 24) ||
      n_out <= 0 || n_out > 64 || n_out > (int64_t)beams * vocab || eos < -1 || eos >= vocab ||
      (finished && eos < 0) || (out_history && (hist_len < 0 || hist_len > (1 << 24))))
    return gfail(c, "beam_select: a size or eos is out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "beam_select");
  // segments: as short as keeps a search at 4096 of them
  int shift = 4;
  while (shift < 10 && (int64_t)beams * (((int64_t)vocab + (1 << shift) - 1) >> shift) > 4096) shift += 2;
  const int segs = (int)(((int64_t)vocab + (1 << shift) - 1) >> shift);
  const int waves = (vocab + kScan - 1) / kScan;
  const int64_t rows = (int64_t)groups * beams, need = rows * (waves * 8 + (int64_t)segs * 4);
  const bool graph = capturing(c->stream);
  if (need > c->beam_cap) {
    if (graph) {
      c->last_error = "beam_select: a captured call needs scratch; make one of its size before";
      return TERMEZO_ERR_STATE;
    }
    if (c->beam_held) c->held.push_back(c->d_beam);
    else if (c->d_beam) (void)hipFree(c->d_beam);
    c->d_beam = nullptr;
    c->beam_cap = 0;
    c->beam_held = false;
    const hipError_t e = hipMalloc(&c->d_beam, (size_t)need);
    if (e != hipSuccess) return hip_status(c, e, "beam_select");
    c->beam_cap = need;
  }
  c->beam_held |= graph;
  BeamArgs a{logits, scores, finished, beams, vocab, n_out, eos, out_scores, out_tokens, out_parents,
             out_finished, history, out_history, hist_len, (float2*)c->d_beam,
             (float*)((char*)c->d_beam + rows * waves * 8), waves, segs, shift};
  // grid.y holds 65535 rows: further ones in launches of their own
  for (int64_t r0 = 0; r0 < rows; r0 += 65535) {
    BeamArgs p = a;
    p.logits += r0 * vocab;
    if (p.finished) p.finished += r0;
    p.part += r0 * waves;
    p.seg += r0 * segs;
    const dim3 grid((unsigned)((waves + 3) / 4), (unsigned)std::min<int64_t>(65535, rows - r0));
    switch (shift) {
      case 4: hipLaunchKernelGGL(k_beam_scan<4>, grid, dim3(256), 0, c->stream, p); break;
      case 6: hipLaunchKernelGGL(k_beam_scan<6>, grid, dim3(256), 0, c->stream, p); break;
      case 8: hipLaunchKernelGGL(k_beam_scan<8>, grid, dim3(256), 0, c->stream, p); break;
      default: hipLaunchKernelGGL(k_beam_scan<10>, grid, dim3(256), 0, c->stream, p);
    }
  }
  hipLaunchKernelGGL(k_beam_pick, dim3((unsigned)groups), dim3(kPick), 0, c->stream, a);
  return hip_status(c, hipGetLastError(), "beam_select");
}

}  // extern "C"
