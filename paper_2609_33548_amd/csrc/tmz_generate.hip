// Choosing the next tokens: the logits of a few rows of hidden states over the embedding, and beam
// search's selection among them.
#include <algorithm>
#include <cmath>
#include <string>

#include "tmz_device.h"
#include "tmz_internal.h"

namespace tmz {

// Logits: a wave per vocabulary row and hidden state.
template <typename T>
__global__ void __launch_bounds__(256) k_logits_plain(const T* x, const T* E, int64_t M, int64_t d,
                                                      int64_t V, float* out) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), m = blockIdx.y;
  if (t >= V) return;
  float acc = 0.0f;
  for (int64_t i = lane; i < d; i += 64) {
    float a, b;
    if constexpr (sizeof(T) == 2) {
      a = bf16_to_f32(x[m * d + i]);
      b = bf16_to_f32(E[t * d + i]);
    } else {
      a = x[m * d + i];
      b = E[t * d + i];
    }
    acc = fmaf(a, b, acc);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, 64);
  if (lane == 0) out[m * V + t] = acc;
}

hipError_t launch_logits(const void* x, const void* E, termezo_dtype dt, int64_t M, int64_t d,
                         int64_t V, float* out, int n_cu, hipStream_t s) {
  const dim3 grid((unsigned)((V + 3) / 4), (unsigned)M);
  if (dt == TERMEZO_BF16)
    hipLaunchKernelGGL(k_logits_plain<uint16_t>, grid, dim3(256), 0, s, (const uint16_t*)x,
                       (const uint16_t*)E, M, d, V, out);
  else
    hipLaunchKernelGGL(k_logits_plain<float>, grid, dim3(256), 0, s, (const float*)x,
                       (const float*)E, M, d, V, out);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Beam selection: a work group per search.  First each beam's log-sum-exp, then n_out rounds that
// each find the best continuation behind the one found before (score descending, then index).
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
};

__device__ __forceinline__ float clean_logit(float x) { return x == x ? x + 0.0f : -INFINITY; }

__global__ void __launch_bounds__(256) k_beam_plain(BeamArgs a) {
  constexpr int kMaxBeams = 64;
  __shared__ double lse[kMaxBeams], rv[4];
  __shared__ int64_t ri[4];
  const int g = blockIdx.x, tid = threadIdx.x, W = a.beams, V = a.vocab;
  for (int b = 0; b < W; ++b) {
    const float* x = a.logits + ((int64_t)g * W + b) * V;
    float m = -INFINITY;
    for (int t = tid; t < V; t += 256) m = fmaxf(m, clean_logit(x[t]));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if ((tid & 63) == 0) rv[tid >> 6] = m;
    __syncthreads();
    m = (float)fmax(fmax(rv[0], rv[1]), fmax(rv[2], rv[3]));
    __syncthreads();
    double s = 0.0;
    for (int t = tid; t < V; t += 256) s += exp((double)clean_logit(x[t]) - (double)m);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((tid & 63) == 0) rv[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) {
      const double l = (double)m + log(rv[0] + rv[1] + rv[2] + rv[3]);
      lse[b] = l > -INFINITY && l < INFINITY ? l : INFINITY;   // no continuations
    }
    __syncthreads();
  }
  double pv = INFINITY;
  int64_t pi = -1;
  for (int r = 0; r < a.n_out; ++r) {
    double bv = -INFINITY;
    int64_t bi = INT64_MAX;
    for (int b = 0; b < W; ++b) {
      const float* x = a.logits + ((int64_t)g * W + b) * V;
      const float sc = a.scores[(int64_t)g * W + b];
      const bool fin = a.finished && a.finished[(int64_t)g * W + b];
      for (int t = tid; t < V; t += 256) {
        double v = fin ? (t == a.eos ? (double)sc : -INFINITY)
                       : lse[b] < INFINITY ? (double)sc + (double)clean_logit(x[t]) - lse[b] : -INFINITY;
        if (!(v == v)) v = -INFINITY;
        const int64_t i = (int64_t)b * V + t;
        const bool later = v < pv || (v == pv && i > pi);
        if (later && (v > bv || (v == bv && i < bi))) {
          bv = v;
          bi = i;
        }
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const double v = __shfl_xor(bv, o, 64);
      const int64_t i = __shfl_xor(bi, o, 64);
      if (v > bv || (v == bv && i < bi)) {
        bv = v;
        bi = i;
      }
    }
    if ((tid & 63) == 0) {
      rv[tid >> 6] = bv;
      ri[tid >> 6] = bi;
    }
    __syncthreads();
    for (int w = 0; w < 4; ++w)
      if (rv[w] > bv || (rv[w] == bv && ri[w] < bi)) {
        bv = rv[w];
        bi = ri[w];
      }
    pv = bv;
    pi = bi;
    const int64_t o = (int64_t)g * a.n_out + r;
    const int b = (int)(bi / V), t = (int)(bi % V);
    if (tid == 0) {
      a.out_scores[o] = (float)bv;
      a.out_tokens[o] = t;
      a.out_parents[o] = b;
      if (a.out_finished)
        a.out_finished[o] = (a.finished && a.finished[(int64_t)g * W + b]) || t == a.eos;
      if (a.out_history) a.out_history[o * (a.hist_len + 1) + a.hist_len] = t;
    }
    if (a.out_history)
      for (int64_t i = tid; i < a.hist_len; i += 256)
        a.out_history[o * (a.hist_len + 1) + i] = a.history[((int64_t)g * W + b) * a.hist_len + i];
    __syncthreads();
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
  BeamArgs a{logits, scores, finished, beams, vocab, n_out, eos, out_scores, out_tokens, out_parents,
             out_finished, history, out_history, hist_len};
  hipLaunchKernelGGL(k_beam_plain, dim3((unsigned)groups), dim3(256), 0, c->stream, a);
  return hip_status(c, hipGetLastError(), "beam_select");
}

}  // extern "C"
