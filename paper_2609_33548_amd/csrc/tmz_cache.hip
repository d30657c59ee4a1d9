// Cache of keys and values in 8 bits and the attention that reads it.
//
// A block is 64 tokens of one key/value head.  Complete blocks are pages: codes u = q + 128 (a
// byte), one step d per block for the keys and one for the values, value = q d.  The tokens behind
// the last complete block lie in tails in the activation type.  A page is written once and never
// again while its group lives, so the beams of a search share pages through a table
// [slot][block] -> page; only tails have one owner each.  A slot's own page of block j is
// tail_of[slot] * max_blocks + j: the beams of a group advance together and a tail has one owner
// at a time, so no two slots write the same page.
//
// The byte order of a page is that of tmz_pages.h.
// Tails are [64][head_dim] for keys and [head_dim][64] for values.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "tmz_device.h"
#include "tmz_internal.h"
#include "tmz_pages.h"

namespace tmz {

constexpr float kStepFloor = 1e-30f;  // a block's largest magnitude is taken as at least this

// What the kernels see of a cache.
struct CacheView {
  uint8_t *kpage, *vpage;
  float2* step;                       // (keys, values) per layer, page and head
  void *ktail, *vtail;                // [layer][2][slot][head][64 x head_dim]
  int32_t *len, *pend, *sel;          // [groups]: length, pending tokens, tail buffer in use
  int32_t *tail_of, *table;
  const float2* rope;                 // [position][head_dim / 2]; null: no rotation
  int32_t* err;
  int32_t groups, beams, width, heads_kv;
  int64_t slots, max_blocks, max_len;

  __device__ int64_t page_head(int layer, int64_t page, int head) const {
    return ((int64_t)layer * slots * max_blocks + page) * heads_kv + head;
  }
  __device__ int64_t tail_head(int layer, int buf, int64_t slot, int head) const {
    return (((int64_t)layer * 2 + buf) * slots + slot) * heads_kv + head;
  }
  __device__ int64_t own_page(int64_t slot, int64_t block) const {
    return (int64_t)tail_of[slot] * max_blocks + block;
  }
};

// A value that no kernel here writes while it is read, at an address that is the same in a wave: by the
// scalar unit.
template <typename V>
__device__ __forceinline__ V scalar_load(const V* p) {
  return *(const __attribute__((address_space(4))) V*)(uintptr_t)p;
}
// Page of a block of a slot with tail `tail`: blocks below the group's length come from the table; those that
// pending tokens complete are the slot's own.
__device__ __forceinline__ int32_t page_of(const CacheView& c, int64_t slot, int32_t tail, int block, int len) {
  return block < len / kBlock ? scalar_load(c.table + slot * c.max_blocks + block)
                              : (int32_t)(tail * c.max_blocks + block);
}

__device__ __forceinline__ float ld_val(const float* p) { return *p; }
__device__ __forceinline__ float ld_val(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void st_val(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_val(uint16_t* p, float v) {
  *p = __builtin_bit_cast(uint16_t, (__bf16)v);
}
__device__ __forceinline__ float as_type(const float*, float v) { return v; }
__device__ __forceinline__ float as_type(const uint16_t*, float v) { return (float)(__bf16)v; }

typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const uint4 r = *(const uint4*)p;
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(w[j] << 16);
    v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load4(const float* p, float* v) {
  const float4 a = *(const float4*)p;
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load4(const uint16_t* p, float* v) {
  const uint2 r = *(const uint2*)p;
  v[0] = __uint_as_float(r.x << 16);
  v[1] = __uint_as_float(r.x & 0xFFFF0000u);
  v[2] = __uint_as_float(r.y << 16);
  v[3] = __uint_as_float(r.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store4(float* p, v4f v) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(uint16_t* p, v4f v) {
  uint2 r;
  r.x = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[0]) |
        ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[1]) << 16);
  r.y = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2]) |
        ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[3]) << 16);
  *(uint2*)p = r;
}

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  store4(p, v4f{v[0], v[1], v[2], v[3]});
  store4(p + 4, v4f{v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j]) |
           ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j + 1]) << 16);
  *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}

// Tokens that an append takes for group g: counts[g], or n; 0 and a deferred error for counts
// outside 0 .. n and for tokens past the end.
__device__ __forceinline__ int append_count(const CacheView& c, int g, int n, const int32_t* counts) {
  const int k = counts ? counts[g] : n;
  if (k < 0 || k > n || (int64_t)c.len[g] + k > c.max_len) {
    if (threadIdx.x == 0) atomicOr(c.err, 16);
    return 0;
  }
  return k;
}
// Queries that attention answers for group g: the pending tokens.
__device__ __forceinline__ int query_count(const CacheView& c, int g, int n, const int32_t* counts) {
  const int k = c.pend[g];
  if (k > n || (counts && counts[g] != k)) {
    if (threadIdx.x == 0) atomicOr(c.err, 16);
    return 0;
  }
  return k;
}

__global__ void __launch_bounds__(256) k_cache_reset(CacheView c, int g0, int g1) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  const int n = (g1 - g0) * c.beams;
  if (i < n) c.tail_of[g0 * c.beams + i] = g0 * c.beams + i;
  if (i < g1 - g0) c.len[g0 + i] = c.pend[g0 + i] = c.sel[g0 + i] = 0;
}

// Rotary table: the angle p base^(-2i/hd) and its functions in fp64, rounded to fp32.
struct RopeFreq {
  double f[64];
};
__global__ void __launch_bounds__(256) k_rope_table(float2* t, int64_t n, int half, RopeFreq w) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n * half) return;
  const double a = (double)(i / half) * w.f[i % half];
  double s, c;
  sincos(a, &s, &c);
  t[i] = make_float2((float)c, (float)s);
}

// ---------------------------------------------------------------------------
// Append: grid blocks, heads, rows.  A work group takes one block of one head; its values go through
// registers once: a thread holds pieces of 8 dims and their partners HD / 2 further (keys, which are rotated and
// rounded to the activation type) and 4 tokens x 8 dims (values).  A complete block takes the largest
// magnitudes over the work group and leaves as a page, put into its byte order in LDS (the values' 16-byte units
// exchanged by their piece of dims, so that a store's lanes fall on different banks); else the new tokens
// go to a tail: the buffer in use when the block had begun, the other one otherwise (so that the
// call can be made again until the tokens are advanced).  Bound by the bytes moved: 8 x 2048 tokens of 5 heads of
// 128 in bf16 19 us (63 MB, 3.2 TB/s), a token of 64 rows 3.4 us.
// ---------------------------------------------------------------------------
// Codes of eight or four values, byte j the j-th.
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d, float s) {
  auto q = [&](float x) __attribute__((always_inline)) {
    return (uint32_t)((int)fminf(fmaxf(__builtin_rintf(x * s), -127.0f), 127.0f) + 128);
  };
  return q(a) | q(b) << 8 | q(c) << 16 | q(d) << 24;
}
// Where the unit of 16 bytes u of a values page lies in LDS.
__device__ __forceinline__ int unit_at(int u) { return u ^ ((u >> 6 & 3) << 1 | (u >> 3 & 1)); }

template <int HD>
struct AppendShared {
  uint4 page[2][kBlock * HD / 16];
  float red[4][2];
};

// The nth block that a row's cnt new tokens touch.
template <typename T, int HD>
__device__ __forceinline__ void append_block(const CacheView& c, int layer, const T* k, const T* v, int n,
                                             int row, int head, int64_t tail, int len, int buf, int cnt,
                                             int nth, AppendShared<HD>& shared) {
  constexpr int PC = HD / 16, KU = kBlock * PC;          // pairs of pieces of a token, of a block
  constexpr int KL = (KU + 255) / 256;
  constexpr int VC = HD / 8, VU = 16 * VC;               // (4 tokens, 8 dims)
  auto& page = shared.page;
  auto& red = shared.red;
  const int tid = threadIdx.x;
  const int64_t blk = len / kBlock + nth;
  const int64_t t0 = blk * kBlock;                       // first token of the block
  const int begun = nth == 0 ? len % kBlock : 0;         // tokens in the tail
  const int end = (int)std::min<int64_t>((int64_t)len + cnt - t0, kBlock);
  const int64_t th = c.tail_head(layer, nth == 0 ? buf : buf ^ 1, tail, head) * (kBlock * HD);
  T* kt = (T*)c.ktail + th;
  T* vt = (T*)c.vtail + th;
  const bool whole = end == kBlock;
  // rows of this block's tokens in the caller's arrays: token t at (t0 - len + t)
  const int64_t rs = (int64_t)c.heads_kv * HD;
  const int64_t base = ((int64_t)row * n + (t0 - len)) * rs + (int64_t)head * HD;
  float ka[KL][8], kb[KL][8], vx[4][8];
#pragma unroll
  for (int x = 0; x < KL; ++x) {
    const int i = x * 256 + tid, t = i / PC, d = i % PC * 8;
    if (KU % 256 != 0 && i >= KU) continue;
    if (t >= begun && t < end) {
      const T* src = k + base + t * rs + d;
      load8(src, ka[x]);
      load8(src + HD / 2, kb[x]);
      if (c.rope) {
        float r[16];
        const float* rp = (const float*)(c.rope + (t0 + t) * (HD / 2) + d);
        load4(rp, r); load4(rp + 4, r + 4); load4(rp + 8, r + 8); load4(rp + 12, r + 12);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float a = ka[x][j], b = kb[x][j];
          ka[x][j] = as_type(src, a * r[2 * j] - b * r[2 * j + 1]);
          kb[x][j] = as_type(src, b * r[2 * j] + a * r[2 * j + 1]);
        }
      }
      if (!whole) {
        store8(kt + t * HD + d, ka[x]);
        store8(kt + t * HD + d + HD / 2, kb[x]);
      }
    } else if (whole) {
      load8(kt + t * HD + d, ka[x]);
      load8(kt + t * HD + d + HD / 2, kb[x]);
    }
  }
  const int vq = tid / VC * 4, vd = tid % VC * 8;        // the thread's tokens and dims
  if (VU == 256 || tid < VU) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = vq + r;
      if (t >= begun && t < end) {
        load8(v + base + t * rs + vd, vx[r]);
      } else if (whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) vx[r][j] = ld_val(vt + (vd + j) * kBlock + t);
      }
    }
    if (!whole) {
      if (vq >= begun && vq + 4 <= end) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          store4(vt + (vd + j) * kBlock + vq, v4f{vx[0][j], vx[1][j], vx[2][j], vx[3][j]});
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (vq + r >= begun && vq + r < end)
#pragma unroll
            for (int j = 0; j < 8; ++j) st_val(vt + (vd + j) * kBlock + vq + r, vx[r][j]);
      }
    }
  }
  if (!whole) return;
  // largest magnitudes; infinity stands for a value that is not finite
  auto mag = [](float m, float x) { return fmaxf(m, fabsf(x) < INFINITY ? fabsf(x) : INFINITY); };
  float mk = 0.0f, mv = 0.0f;
#pragma unroll
  for (int x = 0; x < KL; ++x)
    if (KU % 256 == 0 || x * 256 + tid < KU)
#pragma unroll
      for (int j = 0; j < 8; ++j) mk = mag(mag(mk, ka[x][j]), kb[x][j]);
  if (VU == 256 || tid < VU)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < 8; ++j) mv = mag(mv, vx[r][j]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    mk = fmaxf(mk, __shfl_xor(mk, o, 64));
    mv = fmaxf(mv, __shfl_xor(mv, o, 64));
  }
  if ((tid & 63) == 0) {
    red[tid >> 6][0] = mk;
    red[tid >> 6][1] = mv;
  }
  __syncthreads();
  float scale[2], step[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const float m = fmaxf(fmaxf(fmaxf(red[0][p], red[1][p]), fmaxf(red[2][p], red[3][p])), kStepFloor);
    const bool fine = m < INFINITY;
    scale[p] = fine ? 127.0f * __fdiv_rn(1.0f, m) : 0.0f;
    step[p] = fine ? m * (1.0f / 127.0f) : __builtin_nanf("");
  }
  const bool k_fine = scale[0] > 0.0f, v_fine = scale[1] > 0.0f;
  uint8_t* kp = (uint8_t*)page[0];
  uint8_t* vp = (uint8_t*)page[1];
#pragma unroll
  for (int x = 0; x < KL; ++x) {
    const int i = x * 256 + tid, t = i / PC, d = i % PC * 8;
    if (KU % 256 != 0 && i >= KU) continue;
    auto put = [&](const float (&f)[8], int e) __attribute__((always_inline)) {
      uint2 w = make_uint2(0x80808080u, 0x80808080u);
      if (k_fine)
        w = make_uint2(code4(f[0], f[1], f[2], f[3], scale[0]), code4(f[4], f[5], f[6], f[7], scale[0]));
      *(uint2*)(kp + key_at<HD>(t, e)) = w;
    };
    put(ka[x], d);
    put(kb[x], d + HD / 2);
  }
  if (VU == 256 || tid < VU)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = value_at(vq, vd + j);
      const uint32_t w = v_fine ? code4(vx[0][j], vx[1][j], vx[2][j], vx[3][j], scale[1]) : 0x80808080u;
      *(uint32_t*)(vp + unit_at(at >> 4) * 16 + (at & 15)) = w;
    }
  __syncthreads();
  const int64_t ph = c.page_head(layer, tail * c.max_blocks + blk, head);
  uint4* ko = (uint4*)(c.kpage + ph * (kBlock * HD));
  uint4* vo = (uint4*)(c.vpage + ph * (kBlock * HD));
#pragma unroll
  for (int i = tid; i < kBlock * HD / 16; i += 256) {
    ko[i] = page[0][i];
    vo[i] = page[1][unit_at(i)];
  }
  if (tid == 0) c.step[ph] = make_float2(step[0], step[1]);
}

template <typename T, int HD>
__global__ void __launch_bounds__(256) k_cache_append(CacheView c, int layer, const T* k, const T* v,
                                                      int n, const int32_t* counts) {
  __shared__ AppendShared<HD> shared;
  const int head = blockIdx.y, row = blockIdx.z;
  const int g = row / c.width;
  const int64_t tail = c.tail_of[(int64_t)g * c.beams + row % c.width];
  const int len = c.len[g], buf = c.sel[g], cnt = append_count(c, g, n, counts);
  if (blockIdx.x == 0 && head == 0 && row % c.width == 0 && threadIdx.x == 0) c.pend[g] = cnt;
  if (cnt == 0 || (int64_t)(len / kBlock + blockIdx.x) * kBlock >= (int64_t)len + cnt) return;
  append_block<T, HD>(c, layer, k, v, n, row, head, tail, len, buf, cnt, blockIdx.x, shared);
}

__global__ void __launch_bounds__(64) k_cache_begin(CacheView c, int n, const int32_t* counts) {
  const int cnt = append_count(c, blockIdx.x, n, counts);
  if (threadIdx.x == 0) c.pend[blockIdx.x] = cnt;
}

// The pending tokens join the sequences: own pages enter the table, a crossed block border changes
// the tail buffer.
__global__ void __launch_bounds__(256) k_cache_advance(CacheView c) {
  const int g = blockIdx.x;
  const int len = c.len[g], nl = len + c.pend[g];
  __syncthreads();
  for (int b = 0; b < c.width; ++b) {
    const int64_t slot = (int64_t)g * c.beams + b;
    for (int j = len / kBlock + threadIdx.x; j < nl / kBlock; j += 256)
      c.table[slot * c.max_blocks + j] = (int32_t)c.own_page(slot, j);
  }
  if (threadIdx.x == 0) {
    c.len[g] = nl;
    c.pend[g] = 0;
    if (nl / kBlock != len / kBlock) c.sel[g] ^= 1;
  }
}

// ---------------------------------------------------------------------------
// Reordering.  The first child of a sequence takes its tail over; further children take the tails
// of sequences without children and get a copy of the tokens in it.  Every work group forms the
// same assignment from the parents: tail[b] the tail of new beam b, from[b] the tail to copy into
// it (-1: none).  parents null: all beams continue beam 0.
// ---------------------------------------------------------------------------
constexpr int kMaxBeams = 64;
struct Assignment {
  int parent[kMaxBeams], tail[kMaxBeams], from[kMaxBeams];
};
__device__ __forceinline__ void assign_tails(const CacheView& c, const int32_t* parents, int g,
                                             Assignment& a) {
  if (threadIdx.x == 0) {
    const int W = c.beams;
    const int64_t s0 = (int64_t)g * W;
    unsigned long long used = 0;
    for (int b = 0; b < W; ++b) {
      int p = parents ? parents[s0 + b] : 0;
      if (p < 0 || p >= W) {
        atomicOr(c.err, 32);
        p = b;
      }
      a.parent[b] = p;
      a.tail[b] = -1;
      a.from[b] = -1;
      if (!(used >> p & 1)) a.tail[b] = c.tail_of[s0 + p];
      used |= 1ull << p;
    }
    int spare = 0;
    for (int b = 0; b < W; ++b)
      if (a.tail[b] < 0) {
        while (used >> spare & 1) ++spare;
        a.tail[b] = c.tail_of[s0 + spare++];
        a.from[b] = c.tail_of[s0 + a.parent[b]];
      }
  }
  __syncthreads();
}

template <typename T, int HD>
__global__ void __launch_bounds__(256) k_reorder_tails(CacheView c, const int32_t* parents) {
  __shared__ Assignment a;
  const int layer = blockIdx.x, head = blockIdx.y, g = blockIdx.z;
  const int t = c.len[g] % kBlock;
  if (t == 0) return;
  assign_tails(c, parents, g, a);
  const int buf = c.sel[g];
  constexpr int EPC = 16 / (int)sizeof(T);
  const int vch = (t + EPC - 1) / EPC;                 // 16-byte pieces of a row of values
  for (int b = 0; b < c.beams; ++b) {
    if (a.from[b] < 0) continue;
    const int64_t from = c.tail_head(layer, buf, a.from[b], head) * (kBlock * HD),
                  to = c.tail_head(layer, buf, a.tail[b], head) * (kBlock * HD);
    for (int i = threadIdx.x; i < t * HD / EPC; i += 256)
      ((uint4*)((T*)c.ktail + to))[i] = ((const uint4*)((const T*)c.ktail + from))[i];
    for (int i = threadIdx.x; i < HD * vch; i += 256) {
      const int at = i / vch * (kBlock / EPC) + i % vch;
      ((uint4*)((T*)c.vtail + to))[at] = ((const uint4*)((const T*)c.vtail + from))[at];
    }
  }
}

__global__ void __launch_bounds__(256) k_reorder_table(CacheView c, const int32_t* parents) {
  __shared__ Assignment a;
  const int g = blockIdx.x, W = c.beams;
  assign_tails(c, parents, g, a);
  const int64_t s0 = (int64_t)g * W;
  int32_t old[kMaxBeams];
  for (int64_t j = threadIdx.x; j < c.len[g] / kBlock; j += 256) {   // a thread, a column
#pragma unroll
    for (int b = 0; b < kMaxBeams; ++b)
      if (b < W) old[b] = c.table[(s0 + a.parent[b]) * c.max_blocks + j];
#pragma unroll
    for (int b = 0; b < kMaxBeams; ++b)
      if (b < W) c.table[(s0 + b) * c.max_blocks + j] = old[b];
  }
  if ((int)threadIdx.x < W) c.tail_of[s0 + threadIdx.x] = a.tail[threadIdx.x];
}

// ---------------------------------------------------------------------------
// Values of a range of positions: grid blocks, heads, rows.  A thread takes 4 tokens x 8 dims: keys 8 bytes a
// token, values 4 bytes a dim (from the caches after the first), 8 values a store.  Bound by the stores: the same
// 8 x 2048 tokens to fp32 24 us (84 MB written, 4.4 TB/s with the reads).
// ---------------------------------------------------------------------------
template <typename T, int HD, typename O>
__global__ void __launch_bounds__(256) k_cache_read(CacheView c, int layer, int64_t first, int64_t n,
                                                    O* ko, O* vo) {
  constexpr int VC = HD / 8;
  const int head = blockIdx.y, row = blockIdx.z, tid = threadIdx.x;
  const int g = row / c.width;
  const int64_t slot = (int64_t)g * c.beams + row % c.width;
  const int64_t tail = c.tail_of[slot];
  const int len = c.len[g], total = len + c.pend[g], sel = c.sel[g];
  const int64_t blk = first / kBlock + blockIdx.x, t0 = blk * kBlock;
  const int64_t stop = std::min(first + n, (int64_t)total);
  const int tq = tid / VC * 4, d = tid % VC * 8;
  if (t0 >= stop || tid >= 16 * VC) return;
  const bool coded = t0 + kBlock <= total;
  const int64_t page = !coded ? 0 : blk < len / kBlock ? c.table[slot * c.max_blocks + blk] : tail * c.max_blocks + blk;
  const int64_t ph = c.page_head(layer, page, head);
  const int64_t th = c.tail_head(layer, sel ^ (blk != len / kBlock), tail, head) * (kBlock * HD);
  const float2 step = coded ? c.step[ph] : make_float2(0.0f, 0.0f);
  const int64_t rs = (int64_t)c.heads_kv * HD;
  const int64_t base = ((int64_t)row * n + (t0 - first)) * rs + (int64_t)head * HD + d;
  float kx[4][8], vx[4][8];
  if (coded) {
    const uint8_t* kp = c.kpage + ph * (kBlock * HD);
    const uint8_t* vp = c.vpage + ph * (kBlock * HD);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint2 w = *(const uint2*)(kp + key_at<HD>(tq + r, d));
#pragma unroll
      for (int j = 0; j < 8; ++j)
        kx[r][j] = (float)((int)((j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 255) - 128) * step.x;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t w = *(const uint32_t*)(vp + value_at(tq, d + j));
#pragma unroll
      for (int r = 0; r < 4; ++r) vx[r][j] = (float)((int)(w >> (8 * r) & 255) - 128) * step.y;
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) load8((const T*)c.ktail + th + (tq + r) * HD + d, kx[r]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float x[4];
      load4((const T*)c.vtail + th + (d + j) * kBlock + tq, x);
#pragma unroll
      for (int r = 0; r < 4; ++r) vx[r][j] = x[r];
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t pos = t0 + tq + r;
    if (pos < first || pos >= stop) continue;
    if (ko) store8(ko + base + (tq + r) * rs, kx[r]);
    if (vo) store8(vo + base + (tq + r) * rs, vx[r]);
  }
}

// ---------------------------------------------------------------------------
// Attention of a few queries (up to 32 (query, head) columns of a key/value head) over a long cache.
//
// Scores are formed as S^T = K Q^T and the output as O^T += V^T P^T with 16x16x32 fp16 matrix
// instructions: a lane then holds the scores of one query (column lane % 16) for tokens
// 4 (lane / 16) + r of each 16, which is the operand layout of P^T, so the probabilities never leave
// their registers, and running maximum, sum and rescaling are a lane's own.
//
// Codes are exact in fp16: a byte u beside 0x64 is the fp16 number 1024 + u, less 1152 is q.  A query
// is scaled by a power of two to a largest magnitude in [512, 1024) and rounded to fp16 (2^-11; one
// rounding less than the bf16 that the rotated query would be stored in); fp32 activations take it in
// two parts (2^-22).  Probabilities are scaled to at most 2^15 and rounded to fp16, again in two parts
// for fp32.  Maxima, sums and outputs are fp32.  O is kept in units of a step of the values so
// far: a block's probabilities take the ratio of its step to that one (take_tokens).  The newest tokens, not
// coded yet, pass the same way: scaled by powers of two to magnitudes below 128, bf16 values are exact in
// fp16 and fp32 ones taken in two parts.
//
// A non-finite value makes every query that sees it NaN and no other: a block with such a value has the
// step NaN, which is put into the scores of its visible tokens, and so is a new token whose value row
// is not finite; weights of hidden tokens are zero and so are the value rows they meet.
//
// Bound by the bytes of the pages: two rows of 131000 tokens (5 heads of 128, 336 MB) 62 us, 5.4 TB/s; 64 rows of
// 3000 (249 MB) 61 us from memory, 4.1 TB/s, and 51 us where the 256 MB cache still holds them; the joining of
// their parts 6 and 5 us more.  16 rows of 2000 with 4 and 8 new tokens (16 and 32 columns) 19 and 23 us, join 5.
// ---------------------------------------------------------------------------
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ v4f mma(v8h a, v8h b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight codes (two words) as fp16.
__device__ __forceinline__ v8h codes_f16(uint32_t w0, uint32_t w1) {
  const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
  uint32_t x[4] = {__builtin_amdgcn_perm(0x64646464u, w0, 0x04010400u),
                   __builtin_amdgcn_perm(0x64646464u, w0, 0x04030402u),
                   __builtin_amdgcn_perm(0x64646464u, w1, 0x04010400u),
                   __builtin_amdgcn_perm(0x64646464u, w1, 0x04030402u)};
  v8h r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const v2h h = __builtin_bit_cast(v2h, x[j]) - off;
    r[2 * j] = h[0];
    r[2 * j + 1] = h[1];
  }
  return r;
}

// v in NS parts of fp16.
template <int NS>
__device__ __forceinline__ void split_f16(const float (&v)[8], v8h (&out)[NS]) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const v2h h = __builtin_convertvector((v2f{v[j], v[j + 1]}), v2h);
    out[0][j] = h[0];
    out[0][j + 1] = h[1];
    if constexpr (NS == 2) {
      const v2h l = __builtin_convertvector((v2f{v[j] - (float)h[0], v[j + 1] - (float)h[1]}), v2h);
      out[1][j] = l[0];
      out[1][j + 1] = l[1];
    }
  }
}

// Exponent e with |m| < 2^e (m finite and positive, else 0), within what ldexp keeps normal.
__device__ __forceinline__ int exponent_of(float m) {
  const int e = (int)(__float_as_uint(m) >> 23 & 255) - 126;
  return m > 0.0f ? (e < -100 ? -100 : e) : 0;
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;
}

// Largest and sum over the four lanes of a column.
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// One column's query as operands (dims 32 k + 8 (lane / 16) .. + 7 of part s in f[k][s]): rotated in
// fp32, scaled; the return value turns a product with codes of step 1 into a score times log2(e).
template <typename T, int HD, int NS>
__device__ __forceinline__ float query_operand(const T* q, const float2* rope, float scale,
                                               v8h (&f)[HD / 32][NS]) {
  const int lane = threadIdx.x & 63;
  float x[HD / 32][8];
  float m = 0.0f;
#pragma unroll
  for (int k = 0; k < HD / 32; ++k) {
    const int d = k * 32 + (lane >> 4) * 8;
    const bool low = d < HD / 2;
    if (q) {
      load8(q + d, x[k]);
      if (rope) {
        float o[8], r[16];
        load8(q + (low ? d + HD / 2 : d - HD / 2), o);
        const float* rp = (const float*)(rope + (low ? d : d - HD / 2));
        load4(rp, r); load4(rp + 4, r + 4); load4(rp + 8, r + 8); load4(rp + 12, r + 12);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float a = x[k][j] * r[2 * j], b = o[j] * r[2 * j + 1];
          x[k][j] = low ? a - b : a + b;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[k][j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_abs(x[k][j]));
  }
  const int e = exponent_of(col_max(m)) - 10;
#pragma unroll
  for (int k = 0; k < HD / 32; ++k) {
#pragma unroll
    for (int j = 0; j < 8; ++j)                          // an infinity would leave scores of -inf alone, and no weight
      x[k][j] = fabsf(x[k][j]) < INFINITY ? ldexpf(x[k][j], -e) : __builtin_nanf("");
    split_f16<NS>(x[k], f[k]);
  }
  return ldexpf(scale * kLog2e, e);
}

// Running softmax of a wave over its blocks: NT tiles of 16 columns.
template <int HD, int NT>
struct Running {
  float m[NT], l[NT];                 // l: this lane's tokens only
  v4f o[NT][HD / 16];
  float unit, top;                    // of o: a step of the values so far (0: none); the largest of them
};

// Keeps the compiler to the order written: READS shared-memory reads, then N - 1 times as many again before
// the MFMAS matrix instructions that use the ones before, then the last ones.  (Left to itself it waits for each
// pair of reads: 148 against 136 us for the ragged prompt batch.)
template <int READS, int MFMAS, int N>
__device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
  for (int i = 0; i < N - 1; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    __builtin_amdgcn_sched_group_barrier(0x8, MFMAS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x8, MFMAS, 0);
}

template <int NS>
constexpr float kScaleBits = NS == 1 ? 7.0f : 15.0f;
constexpr float kNearStep = 0x1p-4f, kLostStep = 0x1p-80f;

// Takes TT tiles of 16 tokens in (a block: 4): s[j][t] the products of column tile j with tokens
// 16 t + 4 (lane / 16) + r, step their steps, qf the columns' factors, last[j] the last of the tokens that the
// column sees (hidden: some column does not see them all), bad the lane's tokens whose values are not
// finite, values(d, h, part) the operand of dims 16 d .. and tokens 32 h ...  NV: parts of the values,
// NS: parts of the probabilities.
//
// The weights exp2(s f - m + bits): m is a column's running maximum (fp32 activations, bits 15), or
// lags behind it by up to 8 (bf16, bits 7: at most 2^15 either way), so that o is seldom rescaled (152 -> 149 us
// for the ragged prompt batch, with the sums by dot products).  They take the ratio of the values' step to the
// unit of o as a summand of the exponent (a fused multiply-add a score either way), and their sum takes its
// inverse.  The unit is the largest step so far, but falls to that of a block whose step is below kNearStep of it,
// so that the ratio is never less: the largest weight is then 2^3 at least, and fp16's floor of 2^-25 is 2^-28 of it.
// Rescaled for such falls, o (at most 2^24 tokens x 2^15 x 127 of the largest unit) stays within fp32 down to kLostStep
// of the largest; blocks of still smaller steps (zeros, whose step is 1e-30 / 127, among them) count in l alone.
// The fall costs the prompt batch 118 -> 122 us, 64 rows of 2000 to 4000 tokens none (66.7 -> 65.6); a second set of
// products scaled in fp32 in its place spilled 26 to 140 registers.
template <int TT, int HD, int NT, int NS, int NV, bool AHEAD, typename Values>
__device__ __forceinline__ void take_tokens(Running<HD, NT>& run, v4f (&s)[NT][TT], float2 step,
                                            const float (&qf)[NT], const int (&last)[NT], bool hidden,
                                            uint32_t bad, Values values) {
  constexpr int HH = (TT + 1) / 2;                       // operands of 32 tokens
  const int tok = (threadIdx.x & 63) >> 4 << 2;
  const bool nan = !(step.x < INFINITY) || !(step.y < INFINITY);
  const float vstep = nan ? 0.0f : step.y;
  const bool far = !nan && vstep < run.unit * kNearStep, lost = !nan && vstep < run.top * kLostStep;
  const float unit = lost ? run.unit : far ? vstep : fmaxf(run.unit, vstep);
  const float ru = __builtin_amdgcn_rcpf(unit);
  const float ratio = nan || lost ? 1.0f : vstep * ru;
  const float shrink = unit != run.unit ? run.unit * ru : 1.0f;
  const float lr = __builtin_amdgcn_logf(ratio);         // log2
  const float inverse = __builtin_amdgcn_rcpf(ratio);
  run.unit = unit;
  run.top = fmaxf(run.top, vstep);
  if (nan || bad)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (nan || (bad >> (t * 4 + r) & 1)) s[j][t][r] = __builtin_nanf("");
  float f[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) f[j] = nan ? 1.0f : qf[j] * step.x;
  if (hidden)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      f[j] = fmaxf(f[j], 0x1p-126f);                     // -inf times 0 would be NaN
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t * 16 + tok + r > last[j]) s[j][t][r] = -INFINITY;
    }
  v8h p[NT][HH][NS];
  float al[NT];
  bool same = shrink == 1.0f && !lost;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    float bm = s[j][0][0];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) bm = fmaxf(bm, s[j][t][r]);
    bm = col_max(bm) * f[j];
    const float m = bm > run.m[j] + (15.0f - kScaleBits<NS>) ? bm : run.m[j];
    const float ref = m == -INFINITY ? 0.0f : m;
    al[j] = __builtin_amdgcn_exp2f(run.m[j] - ref);
    run.m[j] = m;
    same = same && al[j] == 1.0f;
    const float off = (kScaleBits<NS> + lr) - ref;
    float sum = 0.0f;
#pragma unroll
    for (int h = 0; h < HH; ++h) {
      float w[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        w[r] = 2 * h + r / 4 < TT ? __builtin_amdgcn_exp2f(fmaf(s[j][2 * h + r / 4 < TT ? 2 * h + r / 4 : 0][r % 4], f[j], off))
                                  : 0.0f;
        if (NS == 2) sum += w[r];
      }
      split_f16<NS>(w, p[j][h]);
      if (NS == 1) {                                     // the sum of the weights as rounded
        const v2h one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
        for (int r = 0; r < 8; r += 2)
          sum = __builtin_amdgcn_fdot2(v2h{p[j][h][0][r], p[j][h][0][r + 1]}, one, sum, false);
      }
    }
    run.l[j] = fmaf(sum, inverse, run.l[j] * al[j]);
    al[j] *= shrink;
  }
  if (!__all(same)) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) run.o[j][d] *= al[j];
    if (lost)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int h = 0; h < HH; ++h)
#pragma unroll
          for (int b = 0; b < NS; ++b) p[j][h][b] = v8h{};
  }
  auto use = [&](v8h v, int d, int h, int a) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int b = 0; b < NS; ++b)
        if (a + b < 2) run.o[j][d] = mma(v, p[j][h][b], run.o[j][d]);
  };
  if constexpr (!AHEAD) {
    __builtin_amdgcn_sched_barrier(0);                   // no conversions of values before: registers
#pragma unroll
    for (int d = 0; d < HD / 16; ++d)
#pragma unroll
      for (int h = 0; h < HH; ++h)
#pragma unroll
        for (int a = 0; a < NV; ++a) use(values(d, h, a), d, h, a);
  } else {                                               // 16 dims are read while those before are used
    v8h v[2][HH];
#pragma unroll
    for (int h = 0; h < HH; ++h) v[0][h] = values(0, h, 0);
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) {
#pragma unroll
      for (int h = 0; h < HH; ++h) {
        if (d + 1 < HD / 16) v[(d + 1) & 1][h] = values(d + 1, h, 0);
      }
#pragma unroll
      for (int h = 0; h < HH; ++h) use(v[d & 1][h], d, h, 0);
    }
    reads_ahead<HH, HH * NT * NS, HD / 16>();
  }
}

// Takes 16 tokens behind the last complete block in, from token t0 of that block on (have: the tokens
// it holds, more than t0), scaled, in NS parts.  A lane loads its rows once, all at a time.
template <typename T, int HD, int NT, int NS>
__device__ __forceinline__ void take_tail(const T* kt, const T* vt, int t0, int have,
                                          const v8h (&qf)[NT][HD / 32][NS], const float (&qs)[NT],
                                          const int (&pos)[NT], int first, Running<HD, NT>& run) {
  const int lane = threadIdx.x & 63;
  float kx[HD / 32][8], vx[HD / 16][4];
  const bool in = t0 + (lane & 15) < have;
#pragma unroll
  for (int k = 0; k < HD / 32; ++k)
    load8(kt + (t0 + (in ? lane & 15 : 0)) * HD + k * 32 + (lane >> 4) * 8, kx[k]);
  const int vt0 = t0 + (lane >> 4) * 4;
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) load4(vt + (d * 16 + (lane & 15)) * kBlock + vt0, vx[d]);
  float km = 0.0f, vm = 0.0f;
  uint32_t bad = 0;
#pragma unroll
  for (int k = 0; k < HD / 32; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) km = fmaxf(km, in ? finite_abs(kx[k][j]) : 0.0f);
#pragma unroll
  for (int d = 0; d < HD / 16; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (vt0 + r >= have) vx[d][r] = 0.0f;
      vm = fmaxf(vm, finite_abs(vx[d][r]));
      if (!(fabsf(vx[d][r]) < INFINITY)) bad |= 1u << r;
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    km = fmaxf(km, __shfl_xor(km, o, 64));
    vm = fmaxf(vm, __shfl_xor(vm, o, 64));
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) bad |= __shfl_xor(bad, o, 64);
  const int ke = exponent_of(km) - 7, ve = exponent_of(vm) - 7;
  v4f s[NT][1];
  int last[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    s[j][0] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    last[j] = pos[j] - first - t0;
  }
#pragma unroll
  for (int k = 0; k < HD / 32; ++k) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      kx[k][j] = !in ? 0.0f : fabsf(kx[k][j]) < INFINITY ? ldexpf(kx[k][j], -ke) : __builtin_nanf("");
    v8h a[NS];
    split_f16<NS>(kx[k], a);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      s[j][0] = mma(a[0], qf[j][k][0], s[j][0]);
      if constexpr (NS == 2) {
        s[j][0] = mma(a[0], qf[j][k][1], s[j][0]);
        s[j][0] = mma(a[1], qf[j][k][0], s[j][0]);
      }
    }
  }
  v8h a[NS];
  take_tokens<1, HD, NT, NS, NS, false>(run, s, make_float2(ldexpf(1.0f, ke), ldexpf(1.0f, ve)), qs, last, true,
                                 bad, [&](int d, int, int part) {
    if (part == 0) {
      float x[8] = {};
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = bad >> r & 1 ? 0.0f : ldexpf(vx[d][r], -ve);
      split_f16<NS>(x, a);
    }
    return a[part];
  });
}

// Work groups of the attention kernels (one or two column tiles; many columns) on a compute unit.
constexpr int kRowsResident1 = 3, kRowsResident2 = 2, kTileResident = 2;

// Blocks that columns below c1 of a row see, its incomplete one among them.
__device__ __forceinline__ int items_of(int len, int cnt, int cols, int c1, int G) {
  const int last = c1 < cols ? (c1 - 1) / G : cnt - 1;   // the last query among them
  return (len + last) / kBlock + 1;
}

// The split of a row's blocks (its last, incomplete one among them) over work groups: how many are
// used and how many blocks each takes.  Attention and the joining of its parts share it.
__device__ __forceinline__ int blocks_per_split(int items, int splits) {
  return (items + splits - 1) / splits;
}

// A wave's NT column tiles from column c0 on: operands, factors and positions.
template <typename T, int HD, int NT, int NS>
__device__ __forceinline__ void load_columns(const CacheView& c, const T* q, int row, int n, int heads,
                                             int head, int len, int cnt, int c0, float scale,
                                             v8h (&qf)[NT][HD / 32][NS], float (&qs)[NT],
                                             int (&pos)[NT]) {
  const int lane = threadIdx.x & 63, G = heads / c.heads_kv, cols = cnt * G;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int col = c0 + j * 16 + (lane & 15);
    const int i = col < cols ? col / G : cnt - 1, hq = col % G;
    pos[j] = len + i;
    const T* qp = col < cols ? q + (((int64_t)row * n + i) * heads + head * G + hq) * HD : nullptr;
    qs[j] = query_operand<T, HD, NS>(qp, c.rope ? c.rope + (int64_t)pos[j] * (HD / 2) : nullptr, scale,
                                     qf[j]);
  }
}

template <int HD, int NT>
__device__ __forceinline__ void start(Running<HD, NT>& run) {
  run.unit = run.top = 0.0f;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    run.m[j] = -INFINITY;
    run.l[j] = 0.0f;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) run.o[j][d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }
}

// Outputs as such, with the sums over all tokens.
template <int HD, int NT>
__device__ __forceinline__ void finish(Running<HD, NT>& run) {
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const float l = run.l[j] = col_sum(run.l[j]);
    const float f = l == 0.0f ? 0.0f : 1.0f / l;         // first: unit / l may be below the normal numbers
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) run.o[j][d] = run.o[j][d] * f * run.unit;
  }
}

// A wave's columns from c0 on: to out, or as a part (nc columns) for k_attend_join.
template <typename T, int HD, int NT>
__device__ __forceinline__ void store_columns(const Running<HD, NT>& run, T* out, float* pp, int nc, int c0,
                                              int p0, int row, int n, int heads, int head, int G, int cols) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int col = c0 + j * 16 + (lane & 15), pc = p0 + j * 16 + (lane & 15), d0 = (lane >> 4) * 4;
    if (col >= cols) continue;
    if (pp) {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) store4(pp + pc * HD + d * 16 + d0, run.o[j][d]);
      if (lane < 16) {
        pp[nc * HD + pc] = run.m[j];
        pp[nc * HD + nc + pc] = run.l[j];
      }
    } else {
      T* op = out + (((int64_t)row * n + col / G) * heads + head * G + col % G) * HD + d0;
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) store4(op + d * 16, run.o[j][d]);
    }
  }
}

// grid: splits, key/value heads, rows.  A wave takes every fourth block of its work group's share.
// APPEND (n = 1): the rows' new tokens are appended first, each by the work group that takes the block it
// falls into.
template <typename T, int HD, int NT, bool APPEND>
__global__ void __launch_bounds__(256, NT == 1 ? kRowsResident1 : kRowsResident2)
    k_attend_rows(CacheView c, int layer, const T* q, const T* k, const T* v, T* out, int n,
                  const int32_t* counts, int heads, float scale, float* part) {
  constexpr int NS = sizeof(T) == 2 ? 1 : 2, NC = 16 * NT;
  struct Joining {
    float o[2][NC][HD + 4], m[2][NC], l[2][NC];
  };
  __shared__ union {
    Joining join;
    AppendShared<HD> append;
  } shared;
  auto& lo = shared.join.o;
  auto& lm = shared.join.m;
  auto& ll = shared.join.l;
  const int head = blockIdx.y, row = blockIdx.z, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = row / c.width;
  const int64_t slot = (int64_t)g * c.beams + row % c.width;
  const int32_t tail = c.tail_of[slot];
  const int len = c.len[g], sel = c.sel[g];
  const int cnt = APPEND ? append_count(c, g, n, counts) : query_count(c, g, n, counts);
  if (APPEND && blockIdx.x == 0 && head == 0 && row % c.width == 0 && threadIdx.x == 0) c.pend[g] = cnt;
  if (cnt == 0) return;
  const int total = len + cnt;
  const int G = heads / c.heads_kv, cols = cnt * G;
  const int full = total / kBlock, items = (total + kBlock - 1) / kBlock;
  const int per = blocks_per_split(items, gridDim.x);
  const int i0 = blockIdx.x * per, i1 = i0 + per < items ? i0 + per : items;
  if (i0 >= i1) return;
  if (APPEND && i1 == items) {                           // the new token's block is the last one
    append_block<T, HD>(c, layer, k, v, n, row, head, tail, len, sel, cnt, 0, shared.append);
    __threadfence_block();
    __syncthreads();
  }
  v8h qf[NT][HD / 32][NS];
  float qs[NT];
  int pos[NT];
  load_columns<T, HD, NT, NS>(c, q, row, n, heads, head, len, cnt, 0, scale, qf, qs, pos);
  Running<HD, NT> run;
  start(run);
  const int ic = i1 < full ? i1 : full;                  // coded blocks end here
  for (int it = i0 + wave; it < ic; it += 4) {
    const int64_t ph = c.page_head(layer, page_of(c, slot, tail, it, len), head);
    int last[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) last[j] = pos[j] - it * kBlock;
    const bool hidden = it * kBlock + kBlock > len + 1;  // some column may not see all of it
    v4f s[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[j][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const uint4* kp = (const uint4*)(c.kpage + ph * (kBlock * HD)) + lane;
    const uint4* vp = (const uint4*)(c.vpage + ph * (kBlock * HD)) + lane;
    uint4 kr[2][HD / 32], vr[HD / 16];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < HD / 32; ++k) kr[p][k] = kp[(p * (HD / 32) + k) * 64];
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) vr[d] = vp[d * 64];
    const float2 step = c.step[ph];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < HD / 32; ++k) {
        const v8h a = codes_f16(kr[p][k].x, kr[p][k].y), b = codes_f16(kr[p][k].z, kr[p][k].w);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int x = 0; x < NS; ++x) {
            s[j][2 * p] = mma(a, qf[j][k][x], s[j][2 * p]);
            s[j][2 * p + 1] = mma(b, qf[j][k][x], s[j][2 * p + 1]);
          }
      }
    take_tokens<4, HD, NT, NS, 1, false>(run, s, step, qs, last, hidden, 0u, [&](int d, int h, int) {
      return h == 0 ? codes_f16(vr[d].x, vr[d].y) : codes_f16(vr[d].z, vr[d].w);
    });
  }
  if (i1 > full && wave * 16 < total - full * kBlock) {  // a wave, 16 of the tokens behind
    const int64_t th = c.tail_head(layer, sel ^ (full != len / kBlock), tail, head) * (kBlock * HD);
    take_tail<T, HD, NT, NS>((const T*)c.ktail + th, (const T*)c.vtail + th, wave * 16,
                             total - full * kBlock, qf, qs, pos, full * kBlock, run);
  }
  // joined in two rounds
  finish(run);
#pragma unroll
  for (int half = 2; half > 0; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int col = j * 16 + (lane & 15);
        if (lane < 16) {
          lm[wave - half][col] = run.m[j];
          ll[wave - half][col] = run.l[j];
        }
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
          *(v4f*)&lo[wave - half][col][d * 16 + (lane >> 4) * 4] = run.o[j][d];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int col = j * 16 + (lane & 15);
        const float m2 = lm[wave][col], l2 = ll[wave][col];
        const float m = fmaxf(run.m[j], m2), ref = m == -INFINITY ? 0.0f : m;
        const float a = run.l[j] * exp2f(run.m[j] - ref), b = l2 * exp2f(m2 - ref);
        const float l = a + b, fa = l == 0.0f ? 0.0f : a / l, fb = l == 0.0f ? 0.0f : b / l;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
          run.o[j][d] = run.o[j][d] * fa + *(v4f*)&lo[wave][col][d * 16 + (lane >> 4) * 4] * fb;
        run.m[j] = m;
        run.l[j] = l;
      }
    }
    __syncthreads();
  }
  if (wave != 0) return;
  float* pp = items <= per ? nullptr :
      part + (((int64_t)row * c.heads_kv + head) * gridDim.x + blockIdx.x) * NC * (HD + 2);
  store_columns<T, HD, NT>(run, out, pp, NC, 0, 0, row, n, heads, head, G, cols);
}

// ---------------------------------------------------------------------------
// Attention of many queries (prompts and their pieces): a work group of four waves takes kTileCols columns
// of a key/value head, 32 a wave, so the blocks that it walks are converted to fp16 once, into
// LDS, for all of them.  Two LDS buffers: while a block is used the next one's codes are on their way
// in registers; the incomplete block passes the same way (bf16).  Four prompts of up to 2000
// tokens, 20 heads of 128 on 5: 122 us, 0.61 PFLOP/s; the matrix cores are busy 27% of it, the vector units 54%
// (exponentials, rescaling and the packing of weights), and waves wait 28%: none is full, since a wave's scores,
// exponentials and value product follow one another and registers leave two waves a SIMD.  fp32: four prompts of
// 1000 77 us (two parts of everything; 8 registers spilled), eight of 512 with heads of 64 19 us, join 12.
// grid (one dimension): key/value heads fastest, then rows, splits, tiles: the longest tiles of all rows first.
// ---------------------------------------------------------------------------
constexpr int kTileCols = 128;
template <typename T, int HD>
__global__ void __launch_bounds__(256, kTileResident) k_attend_tile(CacheView c, int layer, const T* q, T* out, int n,
                                                     const int32_t* counts, int heads, float scale,
                                                     int splits, float* part) {
  constexpr int NS = sizeof(T) == 2 ? 1 : 2, NT = 2, KS = HD / 32;
  constexpr int kPieces = kBlock * HD / 16;              // 16-byte pieces of a page
  constexpr bool kWhole = NS == 1;                       // the incomplete block is taken whole
  __shared__ uint4 lds[2][4 * kPieces];                  // keys [16 tokens][32 dims], values [16 dims][32 tokens]
  __shared__ float tail_max[2][4];
  __shared__ uint32_t tail_bad[2];
  const int units = c.heads_kv * c.groups * c.width, unit = blockIdx.x % units, turn = blockIdx.x / units;
  const int head = unit % c.heads_kv, row = unit / c.heads_kv, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles = gridDim.x / units / splits, tile = tiles - 1 - turn / splits, split = turn % splits;
  const int g = row / c.width;
  const int cnt = query_count(c, g, n, counts);
  const int G = heads / c.heads_kv, cols = cnt * G, c0 = tile * kTileCols;
  if (c0 >= cols) return;
  const int64_t slot = (int64_t)g * c.beams + row % c.width;
  const int32_t tail = c.tail_of[slot];
  const int len = c.len[g], total = len + cnt, full = total / kBlock;
  const int items = items_of(len, cnt, cols, c0 + kTileCols, G);
  const int per = blocks_per_split(items, splits);
  const int i0 = split * per, i1 = i0 + per < items ? i0 + per : items;
  if (i0 >= i1) return;
  const int wc = c0 + wave * 32;                         // the wave's first column
  const int mine = wc < cols ? items_of(len, cnt, cols, wc + 32, G) : 0;   // blocks it needs
  const int c1 = i1 < full ? i1 : full;                  // coded blocks end here
  // pieces of a page a thread moves, and what they are
  constexpr int PL = (kPieces + 255) / 256;
  uint4 kraw[PL], vraw[PL];
  float2 step_next = make_float2(0.0f, 0.0f);
  int32_t page = i0 < c1 ? page_of(c, slot, tail, i0, len) : 0;
  auto fetch = [&](int it) __attribute__((always_inline)) {
    const int64_t ph = c.page_head(layer, page, head);
    const uint4* kp = (const uint4*)(c.kpage + ph * (kBlock * HD));
    const uint4* vp = (const uint4*)(c.vpage + ph * (kBlock * HD));
#pragma unroll
    for (int x = 0; x < PL; ++x) {
      const int i = x * 256 + tid;
      if (kPieces % 256 == 0 || i < kPieces) {
        kraw[x] = kp[i];
        vraw[x] = vp[i];
      }
    }
    const v2f st = scalar_load((const v2f*)(c.step + ph));
    step_next = make_float2(st[0], st[1]);
    if (it + 1 < c1) page = page_of(c, slot, tail, it + 1, len);
  };
  auto place = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < PL; ++x) {
      const int i = x * 256 + tid;
      if (kPieces % 256 == 0 || i < kPieces) {
        // keys: piece (pair p, dims k) holds 16 tokens 2 p and 2 p + 1; values: (dims d) both halves
        const int f = i >> 6, fk = f / KS * 2 * KS + f % KS, fv = 4 * KS + 2 * f;
        lds[buf][fk * 64 + lane] = __builtin_bit_cast(uint4, codes_f16(kraw[x].x, kraw[x].y));
        lds[buf][(fk + KS) * 64 + lane] = __builtin_bit_cast(uint4, codes_f16(kraw[x].z, kraw[x].w));
        lds[buf][fv * 64 + lane] = __builtin_bit_cast(uint4, codes_f16(vraw[x].x, vraw[x].y));
        lds[buf][(fv + 1) * 64 + lane] = __builtin_bit_cast(uint4, codes_f16(vraw[x].z, vraw[x].w));
      }
    }
  };
  // The incomplete block becomes one of the same form (bf16): scaled by powers of two to magnitudes below 128.  Wave w
  // converts the keys of tokens 16 w .. and HD / 4 dims of the values.  (16 tokens at a time in every wave, as fp32 takes
  // them below for want of registers, measured 25 against 15 us for 16 prompts of 63 tokens, 43 against 37 for 6 pieces
  // of 96 behind 1500, and 15 against 16.5 where the block holds 11 tokens.)  Returns the lane's tokens whose values
  // are not finite.
  auto place_tail = [&]() __attribute__((always_inline)) -> uint32_t {
    const int64_t th = c.tail_head(layer, c.sel[g] ^ (full != len / kBlock), tail, head) * (kBlock * HD);
    const int have = total - full * kBlock;
    const T *kt = (const T*)c.ktail + th, *vt = (const T*)c.vtail + th;
    const int t = wave * 16 + (lane & 15), v0 = (lane >> 4) * 4;
    const bool in = t < have;
    uint4 kr[KS];
    uint2 vr[KS][2];
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      kr[x] = *(const uint4*)(kt + (in ? t : 0) * HD + x * 32 + (lane >> 4) * 8);
      const int f = wave * KS + x;                       // dims 16 (f / 2) .., tokens 32 (f % 2) + v0 .. and 16 further
      const T* vp = vt + (f / 2 * 16 + (lane & 15)) * kBlock + f % 2 * 32 + v0;
      vr[x][0] = *(const uint2*)vp;
      vr[x][1] = *(const uint2*)(vp + 16);
    }
    auto key = [&](int x, float (&k)[8]) __attribute__((always_inline)) { load8((const T*)&kr[x], k); };
    auto value = [&](int x, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        load4((const T*)&vr[x][r], v + 4 * r);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((wave * KS + x) % 2 * 32 + v0 + r * 16 + e >= have) v[4 * r + e] = 0.0f;
      }
    };
    float km = 0.0f, vm = 0.0f;
    uint32_t off[2] = {0, 0};                            // tokens 32 i + v0 + .. with a value that is not finite
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      float k[8], v[8];
      key(x, k);
      value(x, v);
      uint32_t b = 0;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (!(fabsf(v[r]) < INFINITY)) b |= 1u << (r / 4 * 16 + r % 4);
        km = fmaxf(km, in ? finite_abs(k[r]) : 0.0f);
        vm = fmaxf(vm, finite_abs(v[r]));
      }
      off[0] |= (wave * KS + x) % 2 ? 0 : b;
      off[1] |= (wave * KS + x) % 2 ? b : 0;
    }
    if (__any(off[0] | off[1])) {
      if (off[0]) atomicOr(&tail_bad[0], off[0] << v0);
      if (off[1]) atomicOr(&tail_bad[1], off[1] << v0);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      km = fmaxf(km, __shfl_xor(km, o, 64));
      vm = fmaxf(vm, __shfl_xor(vm, o, 64));
    }
    if (lane == 0) {
      tail_max[0][wave] = km;
      tail_max[1][wave] = vm;
    }
    __syncthreads();
    km = fmaxf(fmaxf(tail_max[0][0], tail_max[0][1]), fmaxf(tail_max[0][2], tail_max[0][3]));
    vm = fmaxf(fmaxf(tail_max[1][0], tail_max[1][1]), fmaxf(tail_max[1][2], tail_max[1][3]));
    const uint32_t b0 = tail_bad[0] >> v0, b1 = tail_bad[1] >> v0;   // the lane's tokens 16 i + v0 + r: bits 4 i + r
    const uint32_t bad = (b0 & 15) | (b0 >> 12 & 240) | (b1 & 15) << 8 | (b1 >> 12 & 240) << 8;
    const int ke = exponent_of(km) - 7, ve = exponent_of(vm) - 7;
    step_next = make_float2(ldexpf(1.0f, ke), ldexpf(1.0f, ve));
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const int f = wave * KS + x;
      float k[8], v[8];
      key(x, k);
      value(x, v);
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        k[r] = !in ? 0.0f : fabsf(k[r]) < INFINITY ? ldexpf(k[r], -ke) : __builtin_nanf("");
        v[r] = fabsf(v[r]) < INFINITY ? ldexpf(v[r], -ve) : 0.0f;   // its token is NaN by `bad`
      }
      v8h a[1];
      split_f16<1>(k, a);
      lds[0][f * 64 + lane] = __builtin_bit_cast(uint4, a[0]);
      split_f16<1>(v, a);
      lds[0][(4 * KS + f) * 64 + lane] = __builtin_bit_cast(uint4, a[0]);
    }
    return bad;
  };
  // the first block is on its way while the queries are
  if (i0 < c1) fetch(i0);
  v8h qf[NT][KS][NS];
  float qs[NT];
  int pos[NT];
  load_columns<T, HD, NT, NS>(c, q, row, n, heads, head, len, cnt, wc, scale, qf, qs, pos);
  Running<HD, NT> run;
  start(run);
  if (kWhole && tid < 2) tail_bad[tid] = 0;
  if (i0 < c1) place(0);
  __syncthreads();
  auto use_block = [&](int it, int buf, float2 step, uint32_t bad) __attribute__((always_inline)) {
    int last[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) last[j] = pos[j] - it * kBlock;
    // a tile's operands are read while the one before is used
    v4f s[NT][4];
    v8h a[2][KS];
    auto read_keys = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < KS; ++k) a[t & 1][k] = __builtin_bit_cast(v8h, lds[buf][(t * KS + k) * 64 + lane]);
    };
    read_keys(0);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (t < 3) read_keys(t + 1);
#pragma unroll
      for (int j = 0; j < NT; ++j) s[j][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int x = 0; x < NS; ++x) s[j][t] = mma(a[t & 1][k], qf[j][k][x], s[j][t]);
    }
    reads_ahead<KS, KS * NT * NS, 4>();
    // the wave's first column sees the fewest tokens
    const bool hidden = it * kBlock + kBlock > len + wc / G + 1;
    take_tokens<4, HD, NT, NS, 1, true>(run, s, step, qs, last, hidden, bad, [&](int d, int h, int) {
      return __builtin_bit_cast(v8h, lds[buf][(4 * KS + 2 * d + h) * 64 + lane]);
    });
  };
  for (int it = i0; it < c1; ++it) {
    const int buf = (it - i0) & 1;
    const float2 step = step_next;
    if (it + 1 < c1) fetch(it + 1);
    if (it < mine) use_block(it, buf, step, 0u);
    if (it + 1 < c1) place(buf ^ 1);
    __syncthreads();
  }
  if (i1 > full) {
    if constexpr (kWhole) {
      const uint32_t bad = place_tail();
      __syncthreads();
      if (full < mine) use_block(full, 0, step_next, bad);
    } else if (full < mine) {
      const int64_t th = c.tail_head(layer, c.sel[g] ^ (full != len / kBlock), tail, head) * (kBlock * HD);
      const int have = total - full * kBlock;
#pragma unroll 1
      for (int t0 = 0; t0 < have; t0 += 16)
        take_tail<T, HD, NT, NS>((const T*)c.ktail + th, (const T*)c.vtail + th, t0, have, qf, qs, pos,
                                 full * kBlock, run);
    }
  }
  if (wc >= cols) return;
  finish(run);
  float* pp = items <= per ? nullptr :
      part + ((((int64_t)row * c.heads_kv + head) * tiles + tile) * splits + split) * kTileCols * (HD + 2);
  store_columns<T, HD, NT>(run, out, pp, kTileCols, wc, wave * 32, row, n, heads, head, G, cols);
}

// Joins the parts of a column.  JW = 4: a work group per column, its waves take every fourth part; JW = 1: a
// wave per column.  A lane takes two dims.
template <typename T, int HD, int JW>
__global__ void __launch_bounds__(256) k_attend_join(CacheView c, const float* part, T* out, int n,
                                                     const int32_t* counts, int heads, int splits,
                                                     int nc, int tiles) {
  __shared__ float lo[JW][HD], ll[JW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, head = blockIdx.y, row = blockIdx.z;
  const int g = row / c.width;
  const int cnt = query_count(c, g, n, counts);
  const int G = heads / c.heads_kv, cols = cnt * G, col = JW == 4 ? blockIdx.x : blockIdx.x * 4 + wave;
  if (col >= cols) return;                               // whole work group, or whole wave
  const int tile = col / nc, pc = col % nc;
  const int items = items_of(c.len[g], cnt, cols, (tile + 1) * nc, G), per = blocks_per_split(items, splits);
  if (items <= per) return;                              // written already
  const int used = (items + per - 1) / per;
  const int64_t stride = (int64_t)nc * (HD + 2);
  const float* pp = part + (((int64_t)row * c.heads_kv + head) * tiles + tile) * splits * stride;
  float m = -INFINITY;                                   // of all parts, in every wave
  for (int s = lane; s < used; s += 64) m = fmaxf(m, pp[s * stride + nc * HD + pc]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float ref = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, a0 = 0.0f, a1 = 0.0f;
  const bool mine = 2 * lane < HD;
#pragma unroll 8
  for (int s = JW == 4 ? wave : 0; s < used; s += JW) {
    const float* q = pp + s * stride;
    const float w = q[nc * HD + nc + pc] * __builtin_amdgcn_exp2f(q[nc * HD + pc] - ref);
    const float2 o = mine ? *(const float2*)(q + pc * HD + 2 * lane) : make_float2(0.0f, 0.0f);
    l += w;
    a0 = fmaf(w, o.x, a0);
    a1 = fmaf(w, o.y, a1);
  }
  T* op = out + (((int64_t)row * n + col / G) * heads + head * G + col % G) * HD;
  if (JW == 1) {
    if (mine) {
      st_val(op + 2 * lane, a0 / l);
      st_val(op + 2 * lane + 1, a1 / l);
    }
    return;
  }
  if (mine) *(float2*)&lo[wave][2 * lane] = make_float2(a0, a1);
  if (lane == 0) ll[wave] = l;
  __syncthreads();
  const int e = threadIdx.x;
  if (e < HD) {
    float v = 0.0f, t = 0.0f;
#pragma unroll
    for (int w = 0; w < JW; ++w) {
      v += lo[w][e];
      t += ll[w];
    }
    st_val(op + e, v / t);
  }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
namespace {

CacheView view_of(const termezo_kvcache* c) {
  CacheView v;
  v.kpage = c->kpage;
  v.vpage = c->vpage;
  v.step = c->step;
  v.ktail = c->ktail;
  v.vtail = c->vtail;
  v.len = c->len;
  v.pend = c->pend;
  v.sel = c->sel;
  v.tail_of = c->tail_of;
  v.table = c->table;
  v.rope = c->rope;
  v.err = c->ctx->d_err;
  v.groups = c->cfg.groups;
  v.beams = c->cfg.beams;
  v.width = c->width;
  v.heads_kv = c->cfg.n_kv_heads;
  v.slots = c->slots;
  v.max_blocks = c->max_blocks;
  v.max_len = c->cfg.max_len;
  return v;
}

// f(T(), HD) with the cache's activation type and head size.
#define TMZ_CACHE_TYPES(c, CALL)                                   \
  if ((c)->cfg.act_dtype == TERMEZO_BF16) {                        \
    if ((c)->cfg.head_dim == 64) { CALL(uint16_t, 64); }           \
    else if ((c)->cfg.head_dim == 96) { CALL(uint16_t, 96); }      \
    else { CALL(uint16_t, 128); }                                  \
  } else {                                                         \
    if ((c)->cfg.head_dim == 64) { CALL(float, 64); }              \
    else if ((c)->cfg.head_dim == 96) { CALL(float, 96); }         \
    else { CALL(float, 128); }                                     \
  }

// Work groups over a row's tokens, for `units` rows x heads: as many as run at a time (`resident` on a compute
// unit), but at least a block for each of a work group's four waves at max_len.  The kernels divide
// the tokens that there are, so no length is known here.  One round of work groups measured best: 64 rows of
// 2000 to 4000 tokens, 5 heads of 128: 49 us at 768 work groups in all, 53 at 1024, 53 at 2048; two
// rows of 131000: 62, 75, 72 us.
int token_splits(const termezo_kvcache* c, int64_t units, int resident) {
  const int64_t groups = (int64_t)resident * c->ctx->n_cu;
  return (int)std::max<int64_t>(1, std::min((c->max_blocks + 3) / 4, groups / units));
}

int64_t rows_of(const termezo_kvcache* c) { return (int64_t)c->cfg.groups * c->width; }

// Few parts (8 and less; measured: 5 parts of 18432 columns of 96 19.6 us with four waves a column) leave
// a column's further waves idle.
template <typename T, int HD>
void join(const termezo_kvcache* c, const CacheView& w, T* out, int n, const int32_t* counts, int splits,
          int nc, int tiles, hipStream_t s) {
  const int Hkv = c->cfg.n_kv_heads, cols = n * (c->cfg.n_heads / Hkv);
  const dim3 grid((unsigned)(splits > 8 ? cols : (cols + 3) / 4), (unsigned)Hkv, (unsigned)rows_of(c));
  if (splits > 8)
    hipLaunchKernelGGL((k_attend_join<T, HD, 4>), grid, dim3(256), 0, s, w, c->part, out, n, counts,
                       c->cfg.n_heads, splits, nc, tiles);
  else
    hipLaunchKernelGGL((k_attend_join<T, HD, 1>), grid, dim3(256), 0, s, w, c->part, out, n, counts,
                       c->cfg.n_heads, splits, nc, tiles);
}

}  // namespace

hipError_t cache_append_on(termezo_kvcache* c, int layer, const void* k, const void* v, int64_t n,
                           const int32_t* counts, hipStream_t s) {
  const CacheView w = view_of(c);
  // blocks that n tokens can touch from any place in a block
  const unsigned nb = (unsigned)((n + kBlock - 2) / kBlock + 1);
  const dim3 grid(nb, (unsigned)c->cfg.n_kv_heads, (unsigned)rows_of(c));
#define TMZ_CALL(T, HD)                                                                         \
  hipLaunchKernelGGL((k_cache_append<T, HD>), grid, dim3(256), 0, s, w, layer, (const T*)k,      \
                     (const T*)v, (int)n, counts)
  TMZ_CACHE_TYPES(c, TMZ_CALL)
#undef TMZ_CALL
  return hipGetLastError();
}

hipError_t cache_attention_on(termezo_kvcache* c, int layer, const void* q, const void* k,
                              const void* v, int64_t n, const int32_t* counts, void* out,
                              hipStream_t s) {
  const int64_t group = c->cfg.n_heads / c->cfg.n_kv_heads;
  if (k && (n > 1 || group > 32)) {
    const hipError_t e = cache_append_on(c, layer, k, v, n, counts, s);
    if (e != hipSuccess) return e;
    k = nullptr;
    counts = nullptr;                                  // attention takes the pending counts
  }
  const CacheView w = view_of(c);
  const int H = c->cfg.n_heads, Hkv = c->cfg.n_kv_heads;
  const float scale = (float)(1.0 / std::sqrt((double)c->cfg.head_dim));
  const int64_t cols = n * group, rows = rows_of(c);
  if (cols <= 32) {
    const int nt = cols <= 16 ? 1 : 2;
    const int splits = token_splits(c, rows * Hkv, nt == 1 ? kRowsResident1 : kRowsResident2);
    const dim3 grid((unsigned)splits, (unsigned)Hkv, (unsigned)rows);
#define TMZ_ROWS(T, HD, NT, APPEND)                                                            \
  hipLaunchKernelGGL((k_attend_rows<T, HD, NT, APPEND>), grid, dim3(256), 0, s, w, layer,       \
                     (const T*)q, (const T*)k, (const T*)v, (T*)out, (int)n, counts, H, scale, c->part)
#define TMZ_CALL(T, HD)                                                                        \
  if (nt == 1) {                                                                               \
    if (k) TMZ_ROWS(T, HD, 1, true); else TMZ_ROWS(T, HD, 1, false);                           \
  } else {                                                                                     \
    if (k) TMZ_ROWS(T, HD, 2, true); else TMZ_ROWS(T, HD, 2, false);                           \
  }                                                                                            \
  if (splits > 1) join<T, HD>(c, w, (T*)out, (int)n, k ? nullptr : counts, splits, 16 * nt, 1, s)
    TMZ_CACHE_TYPES(c, TMZ_CALL)
#undef TMZ_CALL
#undef TMZ_ROWS
    return hipGetLastError();
  }
  const int tiles = (int)((cols + kTileCols - 1) / kTileCols);
  const int splits = token_splits(c, rows * Hkv * tiles, kTileResident);
  const dim3 grid((unsigned)(Hkv * rows * tiles * splits));
#define TMZ_CALL(T, HD)                                                                         \
  hipLaunchKernelGGL((k_attend_tile<T, HD>), grid, dim3(256), 0, s, w, layer, (const T*)q,       \
                     (T*)out, (int)n, counts, H, scale, splits, c->part);                       \
  if (splits > 1) join<T, HD>(c, w, (T*)out, (int)n, counts, splits, kTileCols, tiles, s)
  TMZ_CACHE_TYPES(c, TMZ_CALL)
#undef TMZ_CALL
  return hipGetLastError();
}

hipError_t cache_begin_on(termezo_kvcache* c, int64_t n, const int32_t* counts, hipStream_t s) {
  hipLaunchKernelGGL(k_cache_begin, dim3((unsigned)c->cfg.groups), dim3(64), 0, s, view_of(c), (int)n,
                     counts);
  return hipGetLastError();
}

hipError_t cache_advance_on(termezo_kvcache* c, hipStream_t s) {
  hipLaunchKernelGGL(k_cache_advance, dim3((unsigned)c->cfg.groups), dim3(256), 0, s, view_of(c));
  return hipGetLastError();
}

}  // namespace tmz

// ===========================================================================
// C ABI
// ===========================================================================
using namespace tmz;

namespace {

termezo_status cfail(termezo_kvcache* c, termezo_status st, const char* msg) {
  c->ctx->last_error = msg;
  return st;
}

termezo_status hip_status(termezo_kvcache* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return TERMEZO_OK;
  (void)hipGetLastError();                               // reported here, not by the next launch
  c->ctx->last_error = std::string(what) + ": " + hipGetErrorString(e);
  return e == hipErrorOutOfMemory ? TERMEZO_ERR_OOM : TERMEZO_ERR_DEVICE;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

void cache_free(termezo_kvcache* c) {
  void* all[] = {c->kpage, c->vpage, c->step, c->ktail, c->vtail, c->len, c->tail_of, c->table,
                 c->rope, c->part};
  for (void* p : all)
    if (p) (void)hipFree(p);
}

termezo_status cache_reset(termezo_kvcache* c, int g0, int g1) {
  const unsigned nb = (unsigned)(((int64_t)(g1 - g0) * c->cfg.beams + 255) / 256);
  hipLaunchKernelGGL(k_cache_reset, dim3(nb), dim3(256), 0, c->stream, view_of(c), g0, g1);
  return hip_status(c, hipGetLastError(), "kvcache_reset");
}

termezo_status check_tokens(termezo_kvcache* c, int32_t layer, const void* a, const void* b, int64_t n,
                            const int32_t* counts, const char* what) {
  if (layer < 0 || layer >= c->cfg.n_layers || n <= 0 || n > c->cfg.max_len || !a || !b ||
      !aligned16(a) || !aligned16(b) || (reinterpret_cast<uintptr_t>(counts) & 3u) != 0) {
    c->ctx->last_error = std::string(what) + ": layer or n out of range, or a null or misaligned pointer";
    return TERMEZO_ERR_INVALID_ARG;
  }
  return TERMEZO_OK;
}

termezo_status cache_reorder(termezo_kvcache* c, const int32_t* parents) {
  const CacheView w = view_of(c);
  const dim3 grid((unsigned)c->cfg.n_layers, (unsigned)c->cfg.n_kv_heads, (unsigned)c->cfg.groups);
#define TMZ_CALL(T, HD) \
  hipLaunchKernelGGL((k_reorder_tails<T, HD>), grid, dim3(256), 0, c->stream, w, parents)
  TMZ_CACHE_TYPES(c, TMZ_CALL)
#undef TMZ_CALL
  hipLaunchKernelGGL(k_reorder_table, dim3((unsigned)c->cfg.groups), dim3(256), 0, c->stream, w, parents);
  return hip_status(c, hipGetLastError(), "kvcache_reorder");
}

}  // namespace

extern "C" {

termezo_status termezo_kvcache_create(termezo_ctx* ctx, const termezo_kvcache_config* cfg,
                                      termezo_kvcache** out) {
  if (!out) return TERMEZO_ERR_INVALID_ARG;
  *out = nullptr;
  if (!ctx || !cfg) return TERMEZO_ERR_INVALID_ARG;
  const termezo_kvcache_config& f = *cfg;
  const int hd = f.head_dim;
  const bool sizes = f.n_layers > 0 && f.n_layers <= 65535 && f.n_heads > 0 && f.n_heads <= 65535 &&
                     f.n_kv_heads > 0 && f.n_heads % f.n_kv_heads == 0 &&
                     (hd == 64 || hd == 96 || hd == 128) && f.groups > 0 && f.beams > 0 &&
                     f.beams <= kMaxBeams && (int64_t)f.groups * f.beams <= 65535 && f.max_len > 0 &&
                     f.max_len <= (int64_t(1) << 24);
  if (!sizes || (f.act_dtype != TERMEZO_F32 && f.act_dtype != TERMEZO_BF16) ||
      !(f.rope_base == 0.0f || (f.rope_base > 1.0f && std::isfinite(f.rope_base)))) {
    ctx->last_error = "kvcache_create: a size, the type or rope_base is out of range";
    return TERMEZO_ERR_INVALID_ARG;
  }
  const int64_t slots = (int64_t)f.groups * f.beams, nblk = (f.max_len + kBlock - 1) / kBlock;
  if (slots * nblk > INT32_MAX) {
    ctx->last_error = "kvcache_create: more than 2^31 - 1 pages";
    return TERMEZO_ERR_INVALID_ARG;
  }
  termezo_kvcache* c = new (std::nothrow) termezo_kvcache();
  if (!c) return TERMEZO_ERR_OOM;
  c->ctx = ctx;
  c->stream = ctx->stream;
  c->device = ctx->device;
  c->cfg = f;
  c->slots = slots;
  c->max_blocks = nblk;
  c->width = 1;
  DeviceScope scope(c->device);
  hipError_t e = scope.err;
  // sizes in doubles first: what no device holds must not wrap around
  const double heads = (double)f.n_layers * slots * f.n_kv_heads, page = (double)kBlock * hd;
  if (e == hipSuccess && heads * nblk * page * 2 > 1e13) e = hipErrorOutOfMemory;
  auto A = [&](void** p, int64_t bytes) {
    if (e == hipSuccess) e = hipMalloc(p, (size_t)bytes);
  };
  if (e == hipSuccess) {
    const int64_t ph = (int64_t)f.n_layers * slots * f.n_kv_heads;
    const int64_t es = f.act_dtype == TERMEZO_BF16 ? 2 : 4;
    A((void**)&c->kpage, ph * nblk * kBlock * hd);
    A((void**)&c->vpage, ph * nblk * kBlock * hd);
    A((void**)&c->step, ph * nblk * 8);
    A(&c->ktail, ph * 2 * kBlock * hd * es);
    A(&c->vtail, ph * 2 * kBlock * hd * es);
    A((void**)&c->len, (int64_t)f.groups * 12);
    A((void**)&c->tail_of, slots * 4);
    A((void**)&c->table, slots * nblk * 4);
    if (f.rope_base > 0.0f) A((void**)&c->rope, f.max_len * (hd / 2) * 8);
    // parts of at most that many work groups (where there are more units nothing is split)
    A((void**)&c->part, (int64_t)ctx->n_cu *
          std::max(std::max(kRowsResident1 * 16, kRowsResident2 * 32), kTileResident * kTileCols) * (hd + 2) * 4);
  }
  termezo_status st = hip_status(c, e, "kvcache_create");
  if (st == TERMEZO_OK) {
    c->pend = c->len + f.groups;
    c->sel = c->pend + f.groups;
    if (c->rope) {
      const int64_t n = f.max_len * (hd / 2);
      RopeFreq w = {};
      for (int i = 0; i < hd / 2; ++i) w.f[i] = std::pow((double)f.rope_base, -2.0 * i / (double)hd);
      hipLaunchKernelGGL(k_rope_table, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, c->stream,
                         c->rope, f.max_len, hd / 2, w);
      st = hip_status(c, hipGetLastError(), "kvcache_create");
    }
    if (st == TERMEZO_OK) st = cache_reset(c, 0, f.groups);
  }
  if (st != TERMEZO_OK) {
    cache_free(c);
    delete c;
    return st;
  }
  *out = c;
  return TERMEZO_OK;
}

void termezo_kvcache_destroy(termezo_kvcache* c) {
  if (!c) return;
  DeviceScope scope(c->device);
  (void)hipStreamSynchronize(c->stream);
  cache_free(c);
  delete c;
}

termezo_status termezo_kvcache_reset(termezo_kvcache* c, int32_t group) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (group < -1 || group >= c->cfg.groups)
    return cfail(c, TERMEZO_ERR_INVALID_ARG, "kvcache_reset: group out of range");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_reset");
  if (group < 0) {
    c->width = 1;
    c->pending = false;
  }
  return cache_reset(c, group < 0 ? 0 : group, group < 0 ? c->cfg.groups : group + 1);
}

termezo_status termezo_kvcache_fork(termezo_kvcache* c) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (c->pending) return cfail(c, TERMEZO_ERR_STATE, "kvcache_fork: appended tokens are pending");
  if (c->width == c->cfg.beams) return cfail(c, TERMEZO_ERR_STATE, "kvcache_fork: every beam is in use");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_fork");
  const termezo_status st = cache_reorder(c, nullptr);
  if (st == TERMEZO_OK) c->width = c->cfg.beams;
  return st;
}

termezo_status termezo_kvcache_append(termezo_kvcache* c, int32_t layer, const void* k, const void* v,
                                      int64_t n, const int32_t* counts) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  const termezo_status st = check_tokens(c, layer, k, v, n, counts, "kvcache_append");
  if (st != TERMEZO_OK) return st;
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_append");
  c->pending = true;
  return hip_status(c, cache_append_on(c, layer, k, v, n, counts, c->stream), "kvcache_append");
}

termezo_status termezo_kvcache_attention(termezo_kvcache* c, int32_t layer, const void* q,
                                         const void* k, const void* v, int64_t n,
                                         const int32_t* counts, void* out) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  termezo_status st = check_tokens(c, layer, q, out, n, counts, "kvcache_attention");
  if (st == TERMEZO_OK && (k || v)) st = check_tokens(c, layer, k, v, n, counts, "kvcache_attention");
  if (st != TERMEZO_OK) return st;
  if (!k && !c->pending)
    return cfail(c, TERMEZO_ERR_STATE, "kvcache_attention: no tokens are pending");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_attention");
  if (k) c->pending = true;
  return hip_status(c, cache_attention_on(c, layer, q, k, v, n, counts, out, c->stream),
                    "kvcache_attention");
}

termezo_status termezo_kvcache_advance(termezo_kvcache* c) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!c->pending) return cfail(c, TERMEZO_ERR_STATE, "kvcache_advance: no tokens are pending");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_advance");
  c->pending = false;
  return hip_status(c, cache_advance_on(c, c->stream), "kvcache_advance");
}

termezo_status termezo_kvcache_reorder(termezo_kvcache* c, const int32_t* parents) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!parents || (reinterpret_cast<uintptr_t>(parents) & 3u) != 0)
    return cfail(c, TERMEZO_ERR_INVALID_ARG, "kvcache_reorder: null or misaligned parents");
  if (c->pending) return cfail(c, TERMEZO_ERR_STATE, "kvcache_reorder: appended tokens are pending");
  if (c->width != c->cfg.beams) return cfail(c, TERMEZO_ERR_STATE, "kvcache_reorder: not forked");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_reorder");
  return cache_reorder(c, parents);
}

termezo_status termezo_kvcache_read(termezo_kvcache* c, int32_t layer, int64_t first, int64_t n,
                                    void* k_out, void* v_out, termezo_dtype dtype) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->cfg.n_layers || first < 0 || n <= 0 || first > c->cfg.max_len - n ||
      (dtype != TERMEZO_F32 && dtype != TERMEZO_BF16) || !aligned16(k_out) || !aligned16(v_out) ||
      (!k_out && !v_out))
    return cfail(c, TERMEZO_ERR_INVALID_ARG, "kvcache_read: an argument is out of range, null or misaligned");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_read");
  const CacheView w = view_of(c);
  const unsigned nb = (unsigned)((first + n - 1) / kBlock - first / kBlock + 1);
  const dim3 grid(nb, (unsigned)c->cfg.n_kv_heads, (unsigned)rows_of(c));
#define TMZ_CALL(T, HD)                                                                          \
  if (dtype == TERMEZO_F32)                                                                      \
    hipLaunchKernelGGL((k_cache_read<T, HD, float>), grid, dim3(256), 0, c->stream, w, layer, first, \
                       n, (float*)k_out, (float*)v_out);                                         \
  else                                                                                           \
    hipLaunchKernelGGL((k_cache_read<T, HD, uint16_t>), grid, dim3(256), 0, c->stream, w, layer, \
                       first, n, (uint16_t*)k_out, (uint16_t*)v_out)
  TMZ_CACHE_TYPES(c, TMZ_CALL)
#undef TMZ_CALL
  return hip_status(c, hipGetLastError(), "kvcache_read");
}

termezo_status termezo_kvcache_lengths(termezo_kvcache* c, int32_t* lengths) {
  if (!c) return TERMEZO_ERR_INVALID_ARG;
  if (!lengths) return cfail(c, TERMEZO_ERR_INVALID_ARG, "kvcache_lengths: null");
  DeviceScope scope(c->device);
  if (scope.err != hipSuccess) return hip_status(c, scope.err, "kvcache_lengths");
  const termezo_status st = termezo_sync(c->ctx);
  if (st != TERMEZO_OK) return st;
  return hip_status(c, hipMemcpy(lengths, c->len, (size_t)c->cfg.groups * 4, hipMemcpyDeviceToHost),
                    "kvcache_lengths");
}

}  // extern "C"
