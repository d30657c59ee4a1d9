// Products with weights in 8-bit integers, a step for each output channel and one for each token:
// out[m][n] = (sum_k q[m][k] c[n][k]) (d_m steps[n]), and the quantiser of both sides.
#include <algorithm>
#include <cmath>
#include <string>

#include "tmz_device.h"
#include "tmz_internal.h"

namespace tmz {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr float kTokenFloor = 1e-5f, kWeightFloor = 1e-30f;
// Codes of tokens lie in rows of whole kPitch bytes, zeros behind K: products of what a weight row is
// followed by then add nothing (integers have no NaN), and no kernel needs a loop of its own for a last
// partial step.
constexpr int64_t kPitch = 128;
__host__ __device__ inline int64_t pitch_of(int64_t K) { return (K + kPitch - 1) / kPitch * kPitch; }

// ---------------------------------------------------------------------------
// Rows in 8 bits: a = max(max |x|, floor), q = rne(x (127 / a)), step a / 127.  One wave a row, 8 values a
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

template <typename T, int C>
__global__ void __launch_bounds__(256) k_rows_i8(const T* __restrict__ x, int64_t M, int64_t K, int64_t pitch,
                                                 float floor, int8_t* __restrict__ q, float* __restrict__ step) {
  const int lane = threadIdx.x & 63;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= M) return;                                    // whole wave
  const T* row = x + m * K;
  const bool held = K <= 512 * C;
  Eight<T> e[C];
  uint32_t a = 0;
  if (held) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int64_t k = (int64_t)i * 512 + lane * 8;
      if (k < K) e[i].load(row + k);
      else e[i].zero();
    }
#pragma unroll
    for (int i = 0; i < C; ++i) a = max(a, e[i].top());
  } else {
    for (int64_t k = lane * 8; k < K; k += 512) {
      Eight<T> f;
      f.load(row + k);
      a = max(a, f.top());
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  const bool fine = a < 0x7F800000u;
  const float top = fmaxf(__uint_as_float(a), floor);
  const float s = fine ? __fdiv_rn(127.0f, top) : 0.0f;
  if (lane == 0) step[m] = fine ? __fdiv_rn(top, 127.0f) : __uint_as_float(0x7FC00000u);
  int8_t* out = q + m * pitch;
  const uint2 none = make_uint2(0u, 0u);
  if (held) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int64_t k = (int64_t)i * 512 + lane * 8;
      if (k < pitch) *(uint2*)(out + k) = fine ? e[i].codes(s) : none;     // zeros behind K
    }
  } else {
    for (int64_t k = lane * 8; k < pitch; k += 512) {
      Eight<T> f;
      f.zero();
      if (k < K) f.load(row + k);
      *(uint2*)(out + k) = fine ? f.codes(s) : none;
    }
  }
}

hipError_t launch_rows_i8(const void* x, termezo_dtype dt, int64_t M, int64_t K, int64_t pitch, float floor,
                          int8_t* q, float* step, hipStream_t s) {
  const dim3 grid((unsigned)((M + 3) / 4));
  if (dt == TERMEZO_BF16)
    hipLaunchKernelGGL((k_rows_i8<uint16_t, 8>), grid, dim3(256), 0, s, (const uint16_t*)x, M, K, pitch, floor, q, step);
  else
    hipLaunchKernelGGL((k_rows_i8<float, 8>), grid, dim3(256), 0, s, (const float*)x, M, K, pitch, floor, q, step);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Output values: acc (d_m steps[n]), each fp32 operation rounded.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *(__bf16*)p = (__bf16)v; }

// Few rows: lane l of a wave loads 16 bytes of weight row l % 16 at byte 16 (l / 16) of a 64-byte step, the
// same piece of token l % 16 is the other operand.  The four waves of a work group share VT x 16 weight rows and
// divide the steps; their sums are joined in LDS.
// grid: tiles of tokens x tiles of weight rows (the former fastest: they meet in the caches).
template <typename TY, int MT, int VT>
__global__ void __launch_bounds__(256) k_linear_rows(const int8_t* __restrict__ q, const float* __restrict__ xstep,
                                                     const int8_t* __restrict__ codes,
                                                     const float* __restrict__ steps, int64_t M, int64_t K,
                                                     int64_t N, TY* __restrict__ out, int mtiles) {
  __shared__ v4i red[3][MT * VT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m0 = (int64_t)(blockIdx.x % mtiles) * 16 * MT, n0 = (int64_t)(blockIdx.x / mtiles) * 16 * VT;
  const int64_t pitch = pitch_of(K);
  const int piece = (lane >> 4) * 16, nsteps = (int)((K + 63) / 64);
  // rows past the end are read as the last one and not stored
  const int8_t *xp[MT], *cp[VT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + 16 * i + (lane & 15);
    xp[i] = q + (m < M ? m : M - 1) * pitch + piece;
  }
#pragma unroll
  for (int j = 0; j < VT; ++j) {
    const int64_t n = n0 + 16 * j + (lane & 15);
    cp[j] = codes + (n < N ? n : N - 1) * K;
  }
  v4i acc[MT][VT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < VT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
  for (int s = wave; s < nsteps; s += 4) {
    // behind K: any weights, the token's codes are 0 there
    const int64_t k = (int64_t)s * 64 + piece < K ? (int64_t)s * 64 + piece : 0;
    v4i a[VT], b[MT];
#pragma unroll
    for (int j = 0; j < VT; ++j) a[j] = *(const v4i*)(cp[j] + k);
#pragma unroll
    for (int i = 0; i < MT; ++i) b[i] = *(const v4i*)(xp[i] + (int64_t)s * 64);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < VT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], b[i], acc[i][j], 0, 0, 0);
  }
  if (wave > 0)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < VT; ++j) red[wave - 1][i * VT + j][lane] = acc[i][j];
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + 16 * i + (lane & 15);
    if (m >= M) continue;
    const float d = xstep[m];
#pragma unroll
    for (int j = 0; j < VT; ++j) {
#pragma unroll
      for (int w = 0; w < 3; ++w) acc[i][j] += red[w][i * VT + j][lane];
      const int64_t n = n0 + 16 * j + (lane >> 4) * 4;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n + r < N) put(out + m * N + n + r, (float)acc[i][j][r] * (d * steps[n + r]));
    }
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
// ---------------------------------------------------------------------------
typedef int v16i __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
constexpr int kStep = 128;
static_assert(kStep == kPitch, "the tokens' codes come in whole steps");

struct __attribute__((packed, aligned(2))) Unit {        // 16 bytes of a row that may begin anywhere
  v4u v;
};

template <typename TY, int BM, int BN, int WM, int WN, int NST, int BPC>
__global__ void __launch_bounds__(64 * (BM / WM) * (BN / WN), BPC * (BM / WM) * (BN / WN) / 4)
    k_linear_tile(const int8_t* __restrict__ q, const float* __restrict__ xstep, const int8_t* __restrict__ codes,
                  const float* __restrict__ steps, int64_t M, int64_t K, int64_t N, TY* __restrict__ out) {
  constexpr int NW = (BM / WM) * (BN / WN), TM = WM / 32, TN = WN / 32, STAGE = (BM + BN) * kStep;
  constexpr int AJ = BM / 8 / NW, BJ = BN / 8 / NW, DJ = AJ + BJ;      // direct loads of a wave and step: 8 rows each
  static_assert(AJ * 8 * NW == BM && BJ * 8 * NW == BN && DJ * (NST - 1) < 64, "tile");
  __shared__ __attribute__((aligned(1024))) int8_t lds[NST * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / (BN / WN), wn = wave % (BN / WN);
  int64_t tm, tn;
  tile_of_block((M + BM - 1) / BM, (N + BN - 1) / BN, tm, tn);
  const int64_t m0 = tm * BM, n0 = tn * BN, pitch = pitch_of(K);
  const int nk = (int)(pitch / kStep);
  const v4i_rsrc arsrc = buffer_of(q + m0 * pitch, (uint32_t)(min((int64_t)BM, M - m0) * pitch));
  const v4i_rsrc brsrc = buffer_of(codes + n0 * K, (uint32_t)(min((int64_t)BN, N - n0) * K));
  uint32_t aoff[AJ], boff[BJ];
#pragma unroll
  for (int j = 0; j < AJ; ++j) {
    const int row = 8 * (AJ * wave + j) + lane / 8;
    aoff[j] = (uint32_t)(row * pitch) + 16 * ((lane % 8) ^ ((row >> 1) & 7));
  }
#pragma unroll
  for (int j = 0; j < BJ; ++j) {
    const int row = 8 * (BJ * wave + j) + lane / 8;
    boff[j] = (uint32_t)(row * K) + 16 * ((lane % 8) ^ ((row >> 1) & 7));
  }
  const uint32_t w = __builtin_amdgcn_readfirstlane(wave);
  auto issue = [&](int kt, int st) __attribute__((always_inline)) {
    const uint32_t k = (uint32_t)kt * kStep, base = lds_offset(lds) + (uint32_t)(st * STAGE);
    // the whole offset in the part that the range check covers
#pragma unroll
    for (int j = 0; j < AJ; ++j) dma16_buf(aoff[j] + k, arsrc, 0u, base + 1024u * (AJ * w + j));
#pragma unroll
    for (int j = 0; j < BJ; ++j) dma16_buf(boff[j] + k, brsrc, 0u, base + (uint32_t)(BM * kStep) + 1024u * (BJ * w + j));
  };
  const int h = lane >> 5, n32 = lane & 31;
  v16i acc[TN][TM];
#pragma unroll
  for (int b = 0; b < TN; ++b)
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][a][r] = 0;
  const int arow = wm * WM + n32, brow = wn * WN + n32;
  v4i af[2][TM], bf[2][TN];
  auto fragments = [&](int st, int ks, int slot) __attribute__((always_inline)) {
    const int8_t* A = lds + st * STAGE;
    const int8_t* B = A + BM * kStep;
    const int c = 4 * h + ks;
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      const int row = brow + 32 * b;
      bf[slot][b] = *(const v4i*)(B + row * kStep + 16 * (c ^ ((row >> 1) & 7)));
    }
#pragma unroll
    for (int a = 0; a < TM; ++a) {
      const int row = arow + 32 * a;
      af[slot][a] = *(const v4i*)(A + row * kStep + 16 * (c ^ ((row >> 1) & 7)));
    }
  };
  auto products = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int b = 0; b < TN; ++b)
        acc[b][a] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[slot][b], af[slot][a], acc[b][a], 0, 0, 0);
  };
  // stages 0 .. NST - 2 on their way, the first one there before the loop
#pragma unroll
  for (int p = 0; p < NST - 1; ++p)
    if (p < nk) issue(p, p);
  if (NST > 2 && nk >= NST - 1) wait_vmcnt_le<(NST - 2) * DJ>(); else __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  fragments(0, 0, 0);
  int cur = 0;
  for (int kt = 0; kt < nk; ++kt) {
    const int into = cur == 0 ? NST - 1 : cur - 1, next = cur == NST - 1 ? 0 : cur + 1;
    // the stage of step kt - 1: every wave had read it before the last barrier
    if (kt + NST - 1 < nk) issue(kt + NST - 1, into);
#pragma unroll
    for (int ks = 0; ks < 3; ++ks) {
      fragments(cur, ks + 1, (ks + 1) & 1);
      products(ks & 1);
    }
    // step kt + 1 has landed (later ones may be on their way); its first fragments are read ahead of this step's last
    // products
    if (NST > 2 && kt + NST - 1 < nk) wait_vmcnt_le<(NST - 2) * DJ>(); else __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (kt + 1 < nk) fragments(next, 0, 0);
    products(1);
    cur = next;
  }
  // outputs: 32 tokens x WN of a wave at a time
  constexpr int UB = 16 / (int)sizeof(TY), UPR = WN / UB, RB = WN * (int)sizeof(TY), PER = 32 * UPR / 64;
  static_assert(NW * 32 * RB <= NST * STAGE, "outputs of a wave in LDS");
  __syncthreads();
  int8_t* stage = lds + wave * 32 * RB;
  const int64_t nw = n0 + wn * WN;
#pragma unroll
  for (int a = 0; a < TM; ++a) {
    const int64_t mw = m0 + wm * WM + 32 * a;
    const int64_t m = mw + n32;
    const float d = xstep[m < M ? m : M - 1];
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * b + 8 * g + 4 * h;          // four outputs from here on
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t n = nw + col + r;
          v[r] = (float)acc[b][a][4 * g + r] * (d * steps[n < N ? n : N - 1]);
        }
        int8_t* at = stage + n32 * RB + 16 * ((col / UB) ^ (n32 % UPR)) + (col % UB) * (int)sizeof(TY);
        if constexpr (sizeof(TY) == 2)
          *(uint2*)at = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        else
          *(float4*)at = make_float4(v[0], v[1], v[2], v[3]);
      }
    // a wave's LDS operations are in order: no barrier
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 64 * i + lane, row = c / UPR, u = c % UPR;
      const int64_t mo = mw + row, no = nw + u * UB;
      const v4u v = *(const v4u*)(stage + row * RB + 16 * (u ^ (row % UPR)));
      if (mo >= M || no >= N) continue;
      TY* p = out + mo * N + no;
      if (no + UB <= N) {
        ((Unit*)p)->v = v;
      } else {
#pragma unroll
        for (int k = 0; k < UB; ++k)
          if (no + k < N) {
            if constexpr (sizeof(TY) == 2) p[k] = (uint16_t)(v[k / 2] >> (16 * (k % 2)));
            else p[k] = __uint_as_float(v[k]);
          }
      }
    }
  }
}

int64_t linear_i8_scratch(int64_t M, int64_t K) { return M * pitch_of(K) + M * 4; }

template <typename TY>
static void linear_as(const int8_t* q, const float* xstep, const int8_t* codes, const float* steps, int64_t M,
                      int64_t K, int64_t N, TY* out, hipStream_t s) {
  auto tiles = [&](int bm, int bn) { return dim3((unsigned)(((M + bm - 1) / bm) * ((N + bn - 1) / bn))); };
#define TMZ_TILE(BM, BN, WM, WN, NST, BPC)                                                                        \
  hipLaunchKernelGGL((k_linear_tile<TY, BM, BN, WM, WN, NST, BPC>), tiles(BM, BN), dim3(64 * (BM / WM) * (BN / WN)), \
                     0, s, q, xstep, codes, steps, M, K, N, out)
  if (M <= 16) {
    hipLaunchKernelGGL((k_linear_rows<TY, 1, 4>), dim3((unsigned)((N + 63) / 64)), dim3(256), 0, s, q, xstep, codes,
                       steps, M, K, N, out, 1);
  } else if (M <= 64) {
    hipLaunchKernelGGL((k_linear_rows<TY, 4, 4>), dim3((unsigned)((N + 63) / 64)), dim3(256), 0, s, q, xstep, codes,
                       steps, M, K, N, out, 1);
  } else if (M <= 1024) {
    TMZ_TILE(128, 128, 64, 64, 3, 1);
  } else {
    TMZ_TILE(256, 256, 128, 64, 2, 1);
  }
#undef TMZ_TILE
}

hipError_t launch_linear_i8(const void* x, termezo_dtype xdt, int64_t M, int64_t K, const int8_t* codes,
                            const float* steps, int64_t N, void* out, termezo_dtype ydt, void* scratch,
                            int n_cu, hipStream_t s) {
  int8_t* q = (int8_t*)scratch;
  float* xstep = (float*)(q + M * pitch_of(K));
  const hipError_t e = launch_rows_i8(x, xdt, M, K, pitch_of(K), kTokenFloor, q, xstep, s);
  if (e != hipSuccess) return e;
  if (ydt == TERMEZO_BF16)
    linear_as(q, xstep, codes, steps, M, K, N, (uint16_t*)out, s);
  else
    linear_as(q, xstep, codes, steps, M, K, N, (float*)out, s);
  return hipGetLastError();
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
  return hip_status(c, launch_rows_i8(w, dtype, N, K, K, kWeightFloor, codes, steps, c->stream), "quantize_rows");
}

termezo_status termezo_linear_i8(termezo_ctx* c, const void* x, termezo_dtype xdt, int64_t M, int64_t K,
                                 const int8_t* codes, const float* steps, int64_t N, void* out, termezo_dtype ydt) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!x || !codes || !steps || !out || !aligned(x, 16) || !aligned(codes, 16) || !aligned(steps, 4) ||
      !aligned(out, 16))
    return refuse(c, "linear_i8: null or misaligned pointer");
  if (!float_type(xdt) || !float_type(ydt) || !sizes_ok(N, K) || M <= 0 || M > (1 << 24))
    return refuse(c, "linear_i8: a size or a type is out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "linear_i8");
  const termezo_status st = scratch_for(c, c->linear, linear_i8_scratch(M, K), "linear_i8");
  if (st != TERMEZO_OK) return st;
  return hip_status(c, launch_linear_i8(x, xdt, M, K, codes, steps, N, out, ydt, c->linear.p, c->n_cu, c->stream),
                    "linear_i8");
}

}  // extern "C"
