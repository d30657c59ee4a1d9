// Products with weights in 8-bit integers, a step for each output channel and one for each token:
// out[m][n] = (sum_k q[m][k] c[n][k]) (d_m steps[n]), and the quantiser of both sides.
#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "tmz_device.h"
#include "tmz_internal.h"

namespace tmz {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr float kTokenFloor = 1e-5f, kWeightFloor = 1e-30f;
// Codes of tokens lie in rows of whole kPitch bytes, zeros behind K: products of what a weight row is
// followed by then add nothing (integers have no NaN), and no kernel needs a loop of its own for a last
// partial step.
// Eight tokens' 128 bytes lie together: a direct load of 1 KB is then one piece of memory.
constexpr int64_t kPitch = 128;
__host__ __device__ inline int64_t pitch_of(int64_t K) { return (K + kPitch - 1) / kPitch * kPitch; }
// Byte of token m and k (pitch: bytes of a token's row, whole kPitch).
__device__ __forceinline__ int64_t token_at(int64_t m, int64_t k, int64_t pitch) {
  return (m >> 3) * 8 * pitch + (k >> 7) * 1024 + (m & 7) * 128 + (k & 127);
}

// ---------------------------------------------------------------------------
// Rows in 8 bits: a = max(max |x|, floor), q = rne(x s) with s = 127 (1 / a), step a / 127.  One wave a row, 8 values a
// lane and load; rows of up to 512 C values stay in registers, longer ones are read twice.  The largest
// magnitude is taken on the bit patterns, where NaN and infinities are above all numbers: such a row has
// codes 0 and the step NaN.  Bound by the bytes of x.
// ---------------------------------------------------------------------------
template <typename T>
struct Eight {                                           // 8 values as loaded
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = ((const uint4*)p)[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void get(float f[8]) const {
    const uint32_t* w = (const uint32_t*)v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 2)
        f[i] = __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
      else
        f[i] = __uint_as_float(w[i]);
    }
  }
  __device__ __forceinline__ uint32_t top() const {      // the largest magnitude's bits
    float f[8];
    get(f);
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return a;
  }
  __device__ __forceinline__ uint2 codes(float s) const {
    float f[8];
    get(f);
    uint32_t o[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      o[i / 4] |= ((uint32_t)(int32_t)__builtin_rintf(f[i] * s) & 0xFFu) << (8 * (i % 4));
    return make_uint2(o[0], o[1]);
  }
};

// One row by W waves (wave: which of them; W > 1: the whole work group): put(k, codes of k .. k + 7) for all k < end
// (zeros from K on); the step in every lane.
template <int C, int W, typename T, typename F>
__device__ __forceinline__ float row_codes(const T* row, int64_t K, int64_t end, float floor, int lane, int wave, F put) {
  constexpr int PASS = 512 * W;
  const int64_t k0 = wave * 512 + lane * 8;
  const bool held = K <= PASS * C;
  Eight<T> e[C];
  uint32_t a = 0;
  if (held) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int64_t k = k0 + i * PASS;
      if (k < K) e[i].load(row + k);
      else e[i].zero();
    }
#pragma unroll
    for (int i = 0; i < C; ++i) a = max(a, e[i].top());
  } else {
    for (int64_t k = k0; k < K; k += PASS) {
      Eight<T> f;
      f.load(row + k);
      a = max(a, f.top());
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  if constexpr (W > 1) {
    __shared__ uint32_t tops[W];
    if (lane == 0) tops[wave] = a;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) a = max(a, tops[i]);
  }
  const bool fine = a < 0x7F800000u;
  const float top = fmaxf(__uint_as_float(a), floor);
  const float s = fine ? 127.0f * __fdiv_rn(1.0f, top) : 0.0f;
  const uint2 none = make_uint2(0u, 0u);
  if (held) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int64_t k = k0 + i * PASS;
      if (k < end) put(k, fine ? e[i].codes(s) : none);
    }
  } else {
    for (int64_t k = k0; k < end; k += PASS) {
      Eight<T> f;
      f.zero();
      if (k < K) f.load(row + k);
      put(k, fine ? f.codes(s) : none);
    }
  }
  return fine ? __fdiv_rn(top, 127.0f) : __uint_as_float(0x7FC00000u);
}

// TOKENS: into the tokens' layout, else rows of K bytes.
// W waves a row: four where the rows are long or do not give every compute unit eight waves (777 x 6912 in fp32
// 11.3 -> 6 us).
template <typename T, int C, int W, bool TOKENS>
__global__ void __launch_bounds__(256) k_rows_i8(const T* __restrict__ x, int64_t M, int64_t K, int64_t pitch,
                                                 float floor, int8_t* __restrict__ q, float* __restrict__ step) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = W > 1 ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  if (m >= M) return;                                    // whole wave
  const float d = row_codes<C, W>(x + m * K, K, TOKENS ? pitch : K, floor, lane, W > 1 ? wave : 0,
                                  [&](int64_t k, uint2 c) __attribute__((always_inline)) {
                                    *(uint2*)(q + (TOKENS ? token_at(m, k, pitch) : m * K + k)) = c;
                                  });
  if (lane == 0 && (W == 1 || wave == 0)) step[m] = d;
}

template <bool TOKENS>
static hipError_t launch_rows_i8(const void* x, termezo_dtype dt, int64_t M, int64_t K, float floor, int8_t* q,
                                 float* step, int n_cu, hipStream_t s) {
  const int64_t pitch = pitch_of(K);
#define TMZ_ROWS(T, C, W)                                                                                          \
  hipLaunchKernelGGL((k_rows_i8<T, C, W, TOKENS>), dim3((unsigned)((W) > 1 ? M : (M + 3) / 4)), dim3(256), 0, s, (const T*)x, \
                     M, K, pitch, floor, q, step)
  // 2^24 rows of four waves would be 2^32 threads, one more than a launch takes
  const bool wide = (K > 4096 && M < (int64_t(1) << 24)) || M < 8 * (int64_t)n_cu;
  if (dt == TERMEZO_BF16) {
    if (wide) TMZ_ROWS(uint16_t, 4, 4); else TMZ_ROWS(uint16_t, 8, 1);
  } else {
    if (wide) TMZ_ROWS(float, 4, 4); else TMZ_ROWS(float, 8, 1);
  }
#undef TMZ_ROWS
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Output values: acc (d_m steps[n]), each fp32 operation rounded.
// ---------------------------------------------------------------------------
struct __attribute__((packed, aligned(4))) Steps {
  float v[4];
};
struct __attribute__((packed, aligned(2))) Half {        // four bf16 of a row that may begin anywhere
  uint32_t v[2];
};
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *(__bf16*)p = (__bf16)v; }

// ---------------------------------------------------------------------------
// Up to 32 tokens: bound by the bytes of the weights, which are read once, straight into matrix operands: lane l of a
// wave loads 16 bytes of weight row l % 16 at byte 16 (l / 16) of a 64-byte step; the same piece of token l % 16 comes from
// LDS, which holds all tokens' codes (rows 16 bytes apart beyond their length: 16 rows' reads fall on all
// banks).  Up to 16 tokens are taken in 8 bits here, by every work group for itself (one launch); more come
// from the quantiser.  Work groups walk the weights, 16 rows at a time, each wave its own (KW = 1) or all of
// them together, dividing the steps (KW = NW, few weight rows); GS steps ahead of the products.
// 1 x 2560 -> 128256: 57 us (5.8 TB/s), 32 x 1536 -> 32003 15, 3 x 256 -> 688 4.2.  Few weight rows are bound by latency (one
// row's loads, the join, and up to 16 tokens the row maxima before them): 1 / 4 / 16 tokens x 2560 -> 2560 5.8 / 6.1 / 8.2 us,
// 6912 -> 2560 12.8 / 14.2 / 22.4, 2560 -> 13824 14.5 / 14.6 / 17.4, whole calls.
// ---------------------------------------------------------------------------
template <typename TX, typename TY, int MT, int KB, int NW, int KW, int GS>
__global__ void __launch_bounds__(64 * NW) k_linear_walk(const TX* __restrict__ x, const int8_t* __restrict__ q,
                                                     const float* __restrict__ xstep, const int8_t* __restrict__ codes,
                                                     const float* __restrict__ steps, int M, int K, int64_t N,
                                                     TY* __restrict__ out) {
  constexpr int TW = NW / KW;                            // tiles at work
  __shared__ __align__(16) int8_t xs[KB * 1024];
  __shared__ float ds[16 * MT];
  __shared__ v4i red[KW > 1 ? NW : 1][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave % KW, tw = wave / KW;
  const int nsteps = (K + 63) / 64, pitch = nsteps * 64 + 16, g16 = (lane >> 4) * 16;
  const int64_t tiles = (N + 15) / 16;
  // this wave's steps: groups of GS, the waves of a tile in turn
  const int groups = (nsteps + GS - 1) / GS;
  auto row_of = [&](int64_t tile) __attribute__((always_inline)) {
    const int64_t n = tile * 16 + (lane & 15);
    return codes + (n < N ? n : N - 1) * K;
  };
  // behind K, and in groups behind the last: any weights, the tokens' codes are 0 there or the products unused
  auto fetch = [&](const int8_t* row, int g, v4i* a) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < GS; ++u) {
      const int k = (g * GS + u) * 64 + g16;
      a[u] = *(const v4i*)(row + (k < K ? k : 0));
    }
  };
  v4i w[2][GS];
  int64_t tile = (int64_t)blockIdx.x * TW + tw;
  const int8_t* row = row_of(tile < tiles ? tile : tiles - 1);
  fetch(row, kw, w[0]);                                  // on its way while the tokens are prepared
  if constexpr (!std::is_same<TX, void>::value) {
    for (int m = wave; m < M; m += NW) {
      const float d = row_codes<8, 1>(x + (int64_t)m * K, K, nsteps * 64, kTokenFloor, lane, 0,
                                   [&](int64_t k, uint2 c) __attribute__((always_inline)) { *(uint2*)(xs + m * pitch + k) = c; });
      if (lane == 0) ds[m] = d;
    }
  } else {
    const int64_t from = pitch_of(K);
    const int pieces = nsteps * 4;
    for (int i = threadIdx.x; i < M * pieces; i += 64 * NW) {
      const int m = i / pieces, c = i - m * pieces;
      *(uint4*)(xs + m * pitch + c * 16) = *(const uint4*)(q + token_at(m, c * 16, from));
    }
    if ((int)threadIdx.x < M) ds[threadIdx.x] = xstep[threadIdx.x];
  }
  __syncthreads();
  int xo[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xo[i] = (16 * i + (lane & 15) < M ? 16 * i + (lane & 15) : M - 1) * pitch + g16;
  const int64_t stride = (int64_t)gridDim.x * TW;
  for (int64_t first = (int64_t)blockIdx.x * TW; first < tiles; first += stride, tile += stride) {
    const bool mine = tile < tiles;                      // whole wave
    v4i acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4i{0, 0, 0, 0};
    const int64_t n = tile * 16 + (lane >> 4) * 4;
    const int8_t* next = row_of(tile + stride < tiles ? tile + stride : tiles - 1);
    auto use = [&](int g, const v4i* a) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < GS; ++u) {
        if (g * GS + u >= nsteps) break;                 // uniform
#pragma unroll
        for (int i = 0; i < MT; ++i)
          acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u], *(const v4i*)(xs + xo[i] + (g * GS + u) * 64), acc[i], 0, 0, 0);
      }
    };
    // two groups in turn, so that registers need no index; behind the last the next tile's first
    int g = kw, slot = 0;
    for (; g < groups; g += 2 * KW) {
      if (g + KW < groups) fetch(row, g + KW, w[1]);
      else fetch(next, kw, w[1]);
      use(g, w[0]);
      if (g + KW >= groups) {
        slot = 1;
        break;
      }
      if (g + 2 * KW < groups) fetch(row, g + 2 * KW, w[0]);
      else fetch(next, kw, w[0]);
      use(g + KW, w[1]);
    }
    if (slot)
#pragma unroll
      for (int u = 0; u < GS; ++u) w[0][u] = w[1][u];
    row = next;
    if constexpr (KW > 1) {
#pragma unroll
      for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
      __syncthreads();
      if (kw == 0)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int v = 1; v < KW; ++v) acc[i] += red[wave + v][i][lane];
    }
    if (mine && kw == 0) {
      float st[4];
      if (n + 3 < N) {
        const Steps f = *(const Steps*)(steps + n);
#pragma unroll
        for (int r = 0; r < 4; ++r) st[r] = f.v[r];
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) st[r] = steps[n + r < N ? n + r : N - 1];
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int m = 16 * i + (lane & 15);
        if (m >= M) continue;
        const float d = ds[m];
        TY* p = out + (int64_t)m * N + n;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = (float)acc[i][r] * (d * st[r]);
        if (n + 3 < N) {
          if constexpr (sizeof(TY) == 4) *(Steps*)p = Steps{{v[0], v[1], v[2], v[3]}};
          else *(Half*)p = Half{{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}};
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (n + r < N) put(p + r, v[r]);
        }
      }
    }
    if constexpr (KW > 1) __syncthreads();               // red is free again
  }
}

// ---------------------------------------------------------------------------
// Many tokens: BM tokens x BN weight rows a work group, K in steps of 128 bytes through a ring of NST stages in LDS that
// direct loads fill (each lane's 16 bytes go from memory to LDS without registers).  Loads of step k + NST - 1
// are issued as step k starts; one barrier a step.  Rows past the ends of the matrices are out of their buffers' range
// and fetch nothing; behind K a weight row is followed by the next one, and the tokens' codes are zeros there.
//   LDS: rows of 128 bytes, 16-byte chunk c of row r at chunk c ^ (r / 2 % 8), so that the fragment reads of
// 16 consecutive rows fall on all banks.
//   v_mfma_i32_32x32x32_i8 with the weights as the first operand: a lane's sixteen sums are one token's, in four
// runs of four neighbouring outputs, which meet in LDS (32 tokens of a wave at a time) so that whole 16-byte units
// go out.  In sub-step ks of a step lane l supplies the chunk 4 (l / 32) + ks of row l % 32 of both operands.
//   Bound by the matrix cores at the clock that they hold: 8192 x 2560 -> 13824 250 us, 2.3 POP/s, busy 66% of the time at
// 1.69 GHz; few tiles by their own loads: 777 x 6912 -> 2560 in fp32 32 us on 140 compute units.
// ---------------------------------------------------------------------------
typedef int v16i __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

typedef uint32_t Unit __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes of a row that may begin anywhere

// SPLIT (TY float): a tile's steps are dealt to `splits` work groups, whose sums go to out [splits][stride] as they are.
template <typename TY, int BM, int BN, int WM, int WN, int NST, int BPC, bool PAST, bool SPLIT>
__global__ void __launch_bounds__(64 * (BM / WM) * (BN / WN), BPC * (BM / WM) * (BN / WN) / 4)
    k_linear_tile(const int8_t* __restrict__ q, const float* __restrict__ xstep, const int8_t* __restrict__ codes,
                  const float* __restrict__ steps, int64_t M, int64_t K, int64_t N, TY* __restrict__ out, int splits,
                  int64_t stride) {
  constexpr int BK = kPitch, NW = (BM / WM) * (BN / WN), TM = WM / 32, TN = WN / 32, STAGE = (BM + BN) * BK;
  constexpr int CH = BK / 16, RPL = 64 / CH, KS = BK / 32;            // chunks a row, rows a direct load, sub-steps
  constexpr int AJ = BM / RPL / NW, BJ = BN / RPL / NW, DJ = AJ + BJ;  // direct loads of a wave and step
  static_assert(AJ * RPL * NW == BM && BJ * RPL * NW == BN && DJ * (NST - 1) < 64, "tile");
  auto turn = [](int row) __attribute__((always_inline)) { return (row >> 1) & 7; };
  __shared__ __attribute__((aligned(1024))) int8_t lds[NST * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / (BN / WN), wn = wave % (BN / WN);
  const int64_t pitch = pitch_of(K);
  const uint32_t nb_m = (uint32_t)((M + BM - 1) / BM), nb_n = (uint32_t)((N + BN - 1) / BN);
  const uint32_t tiles = nb_m * nb_n * (SPLIT ? splits : 1);
  const int nk = (int)((K + BK - 1) / BK);
  // steps of a tile (of its part t % splits, at least one): from, up to
  auto from_step = [&](uint32_t t) __attribute__((always_inline)) { return SPLIT ? (int)(t % splits) * nk / splits : 0; };
  auto to_step = [&](uint32_t t) __attribute__((always_inline)) { return SPLIT ? ((int)(t % splits) + 1) * nk / splits : nk; };
  // This work group's tiles: every XCD takes a contiguous part of the order (groups of kGroupM tile rows, so that the
  // tiles at work on it share rows of both operands in its L2), its work groups take that in turn
  const uint32_t xcd = blockIdx.x % kXcd, groups = (gridDim.x - xcd + kXcd - 1) / kXcd;
  const uint32_t part0 = (uint32_t)xcd_linear(xcd, tiles), part1 = xcd + 1 < kXcd ? (uint32_t)xcd_linear(xcd + 1, tiles) : tiles;
  uint32_t at = part0 + blockIdx.x / kXcd;
  if (at >= part1) return;
  auto place = [&](uint32_t t, int64_t& m, int64_t& n) __attribute__((always_inline)) {
    if (SPLIT) t /= splits;
    const uint32_t span = kGroupM * nb_n, g = t / span, in = t - g * span, gm = min((uint32_t)kGroupM, nb_m - g * kGroupM);
    m = (int64_t)(g * kGroupM + in % gm) * BM;
    n = (int64_t)(in / gm) * BN;
  };
  v4i_rsrc arsrc, brsrc;
  int64_t m0, n0;
  place(at, m0, n0);
  uint32_t aoff[AJ], boff[BJ];
#pragma unroll
  for (int j = 0; j < AJ; ++j) {
    const int row = RPL * (AJ * wave + j) + lane / CH;
    aoff[j] = (uint32_t)token_at(row, 16 * ((lane % CH) ^ turn(row)), pitch);
  }
#pragma unroll
  for (int j = 0; j < BJ; ++j) {
    const int row = RPL * (BJ * wave + j) + lane / CH;
    boff[j] = (uint32_t)(row * K) + 16 * ((lane % CH) ^ turn(row));
  }
  const uint32_t w = __builtin_amdgcn_readfirstlane(wave);
  auto issue = [&](int kt, int st) __attribute__((always_inline)) {
    const uint32_t k = (uint32_t)kt * BK, base = lds_offset(lds) + (uint32_t)(st * STAGE);
    // the whole offset in the part that the range check covers
#pragma unroll
    for (int j = 0; j < AJ; ++j) dma16_buf(aoff[j] + 8 * k, arsrc, 0u, base + 1024u * (AJ * w + j));
#pragma unroll
    for (int j = 0; j < BJ; ++j) dma16_buf(boff[j] + k, brsrc, 0u, base + (uint32_t)(BM * BK) + 1024u * (BJ * w + j));
  };
  const int h = lane >> 5, n32 = lane & 31;
  v16i acc[TN][TM];
  const int arow = wm * WM + n32, brow = wn * WN + n32;
  v4i af[2][TM], bf[2][TN];
  auto fragments = [&](int st, int ks, int slot) __attribute__((always_inline)) {
    const int8_t* A = lds + st * STAGE;
    const int8_t* B = A + BM * BK;
    const int c = KS * h + ks;
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      const int row = brow + 32 * b;
      bf[slot][b] = *(const v4i*)(B + row * BK + 16 * (c ^ turn(row)));
    }
#pragma unroll
    for (int a = 0; a < TM; ++a) {
      const int row = arow + 32 * a;
      af[slot][a] = *(const v4i*)(A + row * BK + 16 * (c ^ turn(row)));
    }
  };
  auto products = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int b = 0; b < TN; ++b)
        acc[b][a] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[slot][b], af[slot][a], acc[b][a], 0, 0, 0);
  };
  // outputs meet in LDS SC columns of 32 tokens at a time: UPR 16-byte units of UB outputs, RB bytes a token
  constexpr int SC = WN < 128 / (int)sizeof(TY) ? WN : 128 / (int)sizeof(TY), UB = 16 / (int)sizeof(TY), UPR = SC / UB;
  constexpr int RB = SC * (int)sizeof(TY), PER = 32 * UPR / 64;
  static_assert(NW * 32 * RB <= STAGE, "outputs of the waves in a stage");
  // The steps of all the work group's tiles are one stream: NST - 1 of them are on their way, across the tiles' ends
  uint32_t ahead = at;                                   // the tile whose steps are being loaded, its next step
  int ahead_k = from_step(at), into = 0, flying = 0;
  bool fresh = true;                                     // none of its steps yet
  auto load = [&]() __attribute__((always_inline)) {
    if (ahead >= part1) return;
    if (fresh) {
      int64_t m, n;
      fresh = false;
      place(ahead, m, n);
      arsrc = buffer_of(q + m * pitch, (uint32_t)(min((int64_t)BM, (M - m + 7) / 8 * 8) * pitch));
      brsrc = buffer_of(codes + n * K, (uint32_t)(min((int64_t)BN, N - n) * K));
    }
    issue(ahead_k, into);
    into = into == NST - 1 ? 0 : into + 1;
    ++flying;
    if (++ahead_k == to_step(ahead)) {
      ahead += groups;
      ahead_k = from_step(ahead);
      fresh = true;
    }
  };
  // the oldest step on its way has landed; NST - 2 later ones may be on theirs
  auto landed = [&]() __attribute__((always_inline)) {
    if (NST > 2 && flying == NST - 1) wait_vmcnt_le<(NST - 2) * DJ>(); else __builtin_amdgcn_s_waitcnt(0);
    --flying;
    __syncthreads();
  };
#pragma unroll
  for (int p = 0; p < NST - 1; ++p) load();
  landed();
  fragments(0, 0, 0);
  int cur = 0;
  for (;; at += groups) {
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][a][r] = 0;
    const int here = to_step(at) - from_step(at);
    for (int kt = 0; kt < here; ++kt) {
      const int next = cur == NST - 1 ? 0 : cur + 1;
      load();                                            // into the stage that every wave had read before the last barrier
#pragma unroll
      for (int ks = 0; ks + 1 < KS; ++ks) {
        // one fragment of the next sub-step, one product, and so on (left alone, the compiler reads each fragment right
        // before its first use and waits for it)
        fragments(cur, ks + 1, (ks + 1) & 1);
        products(ks & 1);
#pragma unroll
        for (int i = 0; i < TM + TN; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          if (i < TM * TN) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        if (TM * TN > TM + TN) __builtin_amdgcn_sched_group_barrier(0x008, TM * TN - TM - TN, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the next step has landed; its first fragments are read ahead of this one's last products
      if (flying > 0) {
        landed();
        fragments(next, 0, 0);
      } else {
        __syncthreads();                                 // the last step of all
      }
      products((KS - 1) & 1);
      __builtin_amdgcn_sched_barrier(0);
      if (kt + 1 < here) cur = next;
    }
    // outputs, through the stage that was just read
    int8_t* stage = lds + cur * STAGE + wave * 32 * RB;
    const int64_t nw = n0 + wn * WN;
    const int64_t mw = m0 + wm * WM;
    float d[TM];
#pragma unroll
    for (int a = 0; a < TM; ++a) {
      const int64_t m = mw + 32 * a + n32;
      d[a] = SPLIT ? 0.0f : xstep[m < M ? m : M - 1];
    }
#pragma unroll
    for (int c0 = 0; c0 < WN; c0 += SC) {
      float st[SC / 32][4][4];
#pragma unroll
      for (int b = 0; b < SC / 32; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int64_t n = nw + c0 + 32 * b + 8 * g + 4 * h;          // four outputs from here on
          if (SPLIT) {
#pragma unroll
            for (int r = 0; r < 4; ++r) st[b][g][r] = 0.0f;
          } else if (n + 3 < N) {
            const Steps f = *(const Steps*)(steps + n);
#pragma unroll
            for (int r = 0; r < 4; ++r) st[b][g][r] = f.v[r];
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) st[b][g][r] = steps[n + r < N ? n + r : N - 1];
          }
        }
#pragma unroll
      for (int a = 0; a < TM; ++a) {
#pragma unroll
        for (int b = 0; b < SC / 32; ++b)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int col = 32 * b + 8 * g + 4 * h;
            float v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int sum = acc[c0 / 32 + b][a][4 * g + r];
              v[r] = SPLIT ? __int_as_float(sum) : (float)sum * (d[a] * st[b][g][r]);
            }
            int8_t* to = stage + n32 * RB + 16 * ((col / UB) ^ (n32 % UPR)) + (col % UB) * (int)sizeof(TY);
            if constexpr (sizeof(TY) == 2)
              *(uint2*)to = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            else
              *(float4*)to = make_float4(v[0], v[1], v[2], v[3]);
          }
        // a wave's LDS operations are in order: no barrier
        v4u o[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int c = 64 * i + lane, row = c / UPR, u = c % UPR;
          o[i] = *(const v4u*)(stage + row * RB + 16 * (u ^ (row % UPR)));
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int c = 64 * i + lane, row = c / UPR, u = c % UPR;
          const int64_t mo = mw + 32 * a + row, no = nw + c0 + u * UB;
          if (mo >= M || no >= N) continue;
          TY* p = out + (SPLIT ? (int64_t)(at % splits) * stride : 0) + mo * N + no;
          if (no + UB <= N) {
            if (PAST) __builtin_nontemporal_store(o[i], (Unit*)p);
            else *(Unit*)p = o[i];
          } else {
#pragma unroll
            for (int k = 0; k < UB; ++k)
              if (no + k < N) {
                if constexpr (sizeof(TY) == 2) p[k] = (uint16_t)(o[i][k / 2] >> (16 * (k % 2)));
                else p[k] = __uint_as_float(o[i][k]);
              }
          }
        }
        __builtin_amdgcn_sched_barrier(0);               // one row tile's values at a time in registers
      }
    }
    if (at + groups >= part1) return;
    __syncthreads();                                     // the stage is free again
    place(at + groups, m0, n0);
    cur = cur == NST - 1 ? 0 : cur + 1;
  }
}

// What a launch of T tiles takes on cu compute units (us): the first tile of a compute unit c0 + l K, further ones a + b K
// each (K in thousands), where T is no multiple of cu the last, partial round counts half of its share and half of a
// whole one.  Fitted to nine weights at 40 to 8192 tokens (rms 9 to 14%); among these the tile with the least estimate is
// within 1% of the best on average, 11% at worst (no other weights were timed with every tile).
struct LinearCost {
  int bm, bn;
  float c0, l, a, b;
};
constexpr LinearCost kLinearBf16[4] = {{256, 256, 6.85f, 8.95f, 6.65f, 16.06f}, {128, 256, 5.56f, 5.71f, 2.18f, 9.58f},
                                       {128, 128, 4.92f, 3.53f, 1.99f, 5.12f}, {64, 64, 4.67f, 1.96f, 0.36f, 1.68f}};
constexpr LinearCost kLinearF32[4] = {{256, 256, 8.23f, 9.05f, 38.11f, 6.72f}, {128, 256, 6.35f, 5.79f, 12.85f, 6.77f},
                                      {128, 128, 5.18f, 3.68f, 4.02f, 4.96f}, {64, 64, 4.62f, 2.10f, 0.70f, 1.68f}};

// The parts' sums [splits][stride] together: out as above, four values a lane (in a row or from one to the next).
template <typename TY>
__global__ void __launch_bounds__(256) k_linear_join(const int* __restrict__ parts, int splits, int64_t stride,
                                                     const float* __restrict__ xstep, const float* __restrict__ steps,
                                                     uint32_t N, uint32_t total, TY* __restrict__ out) {
  const uint32_t e = 4 * (blockIdx.x * 256 + threadIdx.x);
  if (e >= total) return;
  v4i sum = *(const v4i*)(parts + e);                    // stride is a multiple of 4
  for (int p = 1; p < splits; ++p) sum += *(const v4i*)(parts + p * stride + e);
  uint32_t m = e / N, n = e - m * N;
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = e + j < total ? (float)sum[j] * (xstep[m] * steps[n]) : 0.0f;
    if (++n == N) {
      n = 0;
      ++m;
    }
  }
  if (e + 4 <= total) {
    if constexpr (sizeof(TY) == 4) *(float4*)(out + e) = make_float4(v[0], v[1], v[2], v[3]);
    else *(uint2*)(out + e) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (e + j < total) put(out + e + j, v[j]);
  }
}

static int64_t split_stride(int64_t M, int64_t N) { return (M * N + 3) / 4 * 4; }

// Parts of K that few tokens' tiles of 64 x 64 are dealt out in (1: none), where the tiles leave compute units idle
// through long sums; the sums are exact, so that the result does not depend on it.  6912 -> 2560: 40 tokens 20.5 us,
// 7.8 + 3.8 in six parts, 100 tokens 20.6 and 12.0 + 3.9, from 200 on none; 4096 -> 1536: 40 tokens 13.4, 5.1 + 4.6.
static int splits_of(int64_t M, int64_t K, int64_t N, int n_cu) {
  const int64_t T = ((M + 63) / 64) * ((N + 63) / 64), nk = (K + kPitch - 1) / kPitch;
  int best = 1;
  float least = 4.6f + 2.0f * 1e-3f * (float)K;
  if (T > n_cu) return 1;
  for (int S = 2; S <= 8 && S * 4 <= nk; ++S) {
    const float k = 1e-3f * (float)K / (float)S, r = (float)(T * S) / (float)n_cu;
    const float more = 0.5f * (float)((T * S + n_cu - 1) / n_cu - 1) + (r > 1.0f ? 0.5f * (r - 1.0f) : 0.0f);
    const float cost = 4.6f + 2.0f * k + more * (0.4f + 1.7f * k) + 4.0f + (float)((S + 1) * M * N * 4) * 0.33e-6f;
    if (cost < least) {
      best = S;
      least = cost;
    }
  }
  return best;
}

template <typename TY>
static void linear_tiles(const int8_t* q, const float* xstep, const int8_t* codes, const float* steps, int64_t M,
                         int64_t K, int64_t N, TY* out, float* parts, int64_t room, int n_cu, hipStream_t s) {
  auto count = [&](int bm, int bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  const int splits = splits_of(M, K, N, n_cu);
  const int64_t stride = split_stride(M, N);
  if (splits > 1 && splits * stride * 4 <= room) {
    hipLaunchKernelGGL((k_linear_tile<float, 64, 64, 32, 32, 3, 3, false, true>),
                       dim3((unsigned)std::min<int64_t>(count(64, 64) * splits, 3 * (int64_t)n_cu)), dim3(256), 0, s, q, xstep,
                       codes, steps, M, K, N, parts, splits, stride);
    hipLaunchKernelGGL((k_linear_join<TY>), dim3((unsigned)((stride / 4 + 255) / 256)), dim3(256), 0, s, (const int*)parts,
                       splits, stride, xstep, steps, (uint32_t)N, (uint32_t)(M * N), out);
    return;
  }
  // An output of more than the eight L2s hold (4 MB each) goes past them and leaves them to the matrices, where whole
  // 128-byte lines do: 8192 x 2560 -> 13824 295 -> 251 us, 8192 x 6912 -> 2560 180 -> 154 (rows that begin inside
  // lines, 389 x 1536 -> 32003 in fp32: 36 -> 57).
  const bool past = M * N * (int64_t)sizeof(TY) >= int64_t(32) << 20 && N * (int64_t)sizeof(TY) % 128 == 0 &&
                    (reinterpret_cast<uintptr_t>(out) & 127) == 0;
  int best = 0;
  float least = 0.0f;
  for (int t = 0; t < 4; ++t) {
    const LinearCost& c = (sizeof(TY) == 2 ? kLinearBf16 : kLinearF32)[t];
    const int64_t T = count(c.bm, c.bn);
    const float k = 1e-3f * (float)K, r = (float)T / (float)n_cu;
    const float more = 0.5f * (float)((T + n_cu - 1) / n_cu - 1) + (r > 1.0f ? 0.5f * (r - 1.0f) : 0.0f);
    const float cost = c.c0 + c.l * k + more * (c.a + c.b * k);
    if (t == 0 || cost < least) {
      best = t;
      least = cost;
    }
  }
#define TMZ_TILE(BM, BN, WM, WN, NST, BPC, PAST)                                                              \
  hipLaunchKernelGGL((k_linear_tile<TY, BM, BN, WM, WN, NST, BPC, PAST, false>),                                           \
                     dim3((unsigned)std::min<int64_t>(count(BM, BN), (int64_t)BPC * n_cu)),                   \
                     dim3(64 * (BM / WM) * (BN / WN)), 0, s, q, xstep, codes, steps, M, K, N, out, 1, 0)
  switch (best) {
    case 0:
      if (past) TMZ_TILE(256, 256, 128, 64, 2, 1, true);
      else TMZ_TILE(256, 256, 128, 64, 2, 1, false);
      break;
    case 1:
      if (past) TMZ_TILE(128, 256, 64, 64, 3, 1, true);
      else TMZ_TILE(128, 256, 64, 64, 3, 1, false);
      break;
    case 2: TMZ_TILE(128, 128, 64, 32, 4, 1, false); break;
    default: TMZ_TILE(64, 64, 32, 32, 3, 3, false);
  }
#undef TMZ_TILE
}

// Whether the walk takes M tokens of K values, and whether it quantises them itself.
static bool walk_ok(int64_t M, int64_t K) { return M <= 32 && M * ((K + 63) / 64 * 64 + 16) <= 140 * 1024; }
static bool walk_quantises(int64_t M, int64_t K) { return M <= 16 && walk_ok(M, K); }

int64_t linear_i8_scratch(int64_t M, int64_t K) {
  return walk_quantises(M, K) ? 0 : ((M + 7) / 8 * 8 * pitch_of(K) + M * 4 + 15) / 16 * 16;
}
int64_t linear_i8_parts(int64_t M, int64_t K, int64_t N, int n_cu) {
  const int splits = walk_ok(M, K) ? 1 : splits_of(M, K, N, n_cu);
  return splits > 1 ? splits * split_stride(M, N) * 4 : 0;
}

template <typename TX, typename TY>
static void linear_walk(const TX* x, const int8_t* q, const float* xstep, const int8_t* codes, const float* steps,
                        int64_t M, int64_t K, int64_t N, TY* out, int n_cu, hipStream_t s) {
  constexpr int MT = std::is_same<TX, void>::value ? 2 : 1;
  const int64_t tiles = (N + 15) / 16, lds = M * ((K + 63) / 64 * 64 + 16);
#define TMZ_WALK(KB, KW, GRID)                                                                              \
  hipLaunchKernelGGL((k_linear_walk<TX, TY, MT, KB, 8, KW, 8 / (KW > 1 ? 4 : 1)>), dim3((unsigned)(GRID)), dim3(512), 0, s, \
                     x, q, xstep, codes, steps, (int)M, (int)K, N, out)
  if (tiles >= 4 * (int64_t)n_cu) {
    if (lds <= 72 * 1024) TMZ_WALK(72, 1, std::min<int64_t>((tiles + 7) / 8, 2 * n_cu));
    else TMZ_WALK(140, 1, std::min<int64_t>((tiles + 7) / 8, n_cu));
  } else {
    if (lds <= 36 * 1024) TMZ_WALK(36, 8, std::min<int64_t>(tiles, 3 * n_cu));
    else TMZ_WALK(140, 8, std::min<int64_t>(tiles, n_cu));
  }
#undef TMZ_WALK
}

template <typename TY>
static hipError_t linear_as(const void* x, termezo_dtype xdt, int64_t M, int64_t K, const int8_t* codes,
                            const float* steps, int64_t N, TY* out, void* scratch, int64_t bytes, int n_cu, hipStream_t s) {
  if (walk_quantises(M, K)) {
    if (xdt == TERMEZO_BF16)
      linear_walk((const uint16_t*)x, nullptr, nullptr, codes, steps, M, K, N, out, n_cu, s);
    else
      linear_walk((const float*)x, nullptr, nullptr, codes, steps, M, K, N, out, n_cu, s);
    return hipGetLastError();
  }
  int8_t* q = (int8_t*)scratch;
  float* xstep = (float*)(q + (M + 7) / 8 * 8 * pitch_of(K));
  const hipError_t e = launch_rows_i8<true>(x, xdt, M, K, kTokenFloor, q, xstep, n_cu, s);
  if (e != hipSuccess) return e;
  if (walk_ok(M, K))
    linear_walk((const void*)nullptr, q, xstep, codes, steps, M, K, N, out, n_cu, s);
  else
    linear_tiles(q, xstep, codes, steps, M, K, N, out, (float*)((char*)scratch + linear_i8_scratch(M, K)),
                 bytes - linear_i8_scratch(M, K), n_cu, s);
  return hipGetLastError();
}

hipError_t launch_linear_i8(const void* x, termezo_dtype xdt, int64_t M, int64_t K, const int8_t* codes,
                            const float* steps, int64_t N, void* out, termezo_dtype ydt, void* scratch,
                            int64_t bytes, int n_cu, hipStream_t s) {
  if (ydt == TERMEZO_BF16)
    return linear_as(x, xdt, M, K, codes, steps, N, (uint16_t*)out, scratch, bytes, n_cu, s);
  return linear_as(x, xdt, M, K, codes, steps, N, (float*)out, scratch, bytes, n_cu, s);
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
bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool float_type(termezo_dtype t) { return t == TERMEZO_F32 || t == TERMEZO_BF16; }
// Sums of K products of codes (127 x 128 at most) fit int32.
bool sizes_ok(int64_t N, int64_t K) {
  return N > 0 && N <= (1 << 24) && K > 0 && K <= (1 << 17) && K % 16 == 0;
}

}  // namespace

extern "C" {

termezo_status termezo_quantize_rows(termezo_ctx* c, const void* w, termezo_dtype dtype, int64_t N, int64_t K,
                                     int8_t* codes, float* steps) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!w || !codes || !steps || !aligned(w, 16) || !aligned(codes, 16) || !aligned(steps, 4))
    return refuse(c, "quantize_rows: null or misaligned pointer");
  if (!float_type(dtype) || !sizes_ok(N, K)) return refuse(c, "quantize_rows: a size or the type is out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "quantize_rows");
  return hip_status(c, launch_rows_i8<false>(w, dtype, N, K, kWeightFloor, codes, steps, c->n_cu, c->stream), "quantize_rows");
}

termezo_status termezo_linear_i8(termezo_ctx* c, const void* x, termezo_dtype xdt, int64_t M, int64_t K,
                                 const int8_t* codes, const float* steps, int64_t N, void* out, termezo_dtype ydt) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!x || !codes || !steps || !out || !aligned(x, 16) || !aligned(codes, 16) || !aligned(steps, 4) ||
      !aligned(out, 16))
    return refuse(c, "linear_i8: null or misaligned pointer");
  if (!float_type(xdt) || !float_type(ydt) || !sizes_ok(N, K) || M <= 0 || M > (1 << 24) ||
      M > (int64_t(1) << 38) / N)
    return refuse(c, "linear_i8: a size or a type is out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "linear_i8");
  // without room for the parts of a split a captured call does with what there is
  int64_t need = linear_i8_scratch(M, K);
  if (c->linear.cap < need || !capturing(c->stream)) need += linear_i8_parts(M, K, N, c->n_cu);
  const termezo_status st = scratch_for(c, c->linear, need, "linear_i8");
  if (st != TERMEZO_OK) return st;
  return hip_status(c, launch_linear_i8(x, xdt, M, K, codes, steps, N, out, ydt, c->linear.p, c->linear.cap, c->n_cu,
                                        c->stream),
                    "linear_i8");
}

}  // extern "C"
