// Link attention over the blocks that score best, and the summaries that they are scored by.
//
// A block is 64 tokens of a linked chunk (one page; a chunk's last one may be shorter).
//   summary   c_b = mean of the block's K rows of a kv head, rounded to bf16
//   score     s_b = max over the kv head's query heads of <q, c_b>, for each query token
//   taken     the first keep_first and last keep_last blocks, then the best, ties to the lower
//   out, lse  as the link kernels', over the taken blocks and the token's own KV
//
// One workgroup does all of it for one (query token, kv head): scores, selection, attention, in one
// launch. (Scores of a launch of its own, once for all workgroups that share a unit, were not built.)
// Bound by HBM for batches (every summary and every taken block are read once per token and kv
// head), by the chain of its steps for few requests.
//
// Scores are summed in 64 bits. The products of bf16 numbers are exact there and the sums
// nearly: what is taken does not depend on the order of a sum, and equal summaries score
// equal. 256 blocks x 128 x 4 heads take a workgroup 4 us, 720 8.7; the sums always are of four
// heads, also for a group of fewer.
//
// Selection: the scores as order-preserving 64-bit integers in LDS; the smallest one taken is
// found 8 bits at a time from the top (a histogram each; it ends early when a bin is taken
// whole), then the taken blocks are listed in order by a prefix sum over ranges of blocks.
//
// Attention: the eight waves take the listed blocks in turn. bf16: 32-key tiles from memory
// straight into the operand layout of the 16x16x32 matrix instruction, the next tile's loads in
// flight under the current one, up to 16 query heads as columns (as in the decode kernel). fp32:
// the vector ALU, a lane a key for the scores and a lane a value dim for the sums, 4 heads. The
// waves' (m, l, o) merge through LDS. Where the units leave CUs idle, `splits` workgroups share a
// unit's blocks (each scores and selects for itself) and merge_kernel joins their partials.
#include <algorithm>

#include "pic_internal.hpp"

namespace pic {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kT = 32;                  // keys per tile (bf16)
template <typename T>
constexpr int kCols = sizeof(T) == 4 ? 4 : 16;   // query heads of a workgroup
template <typename T>
int col_blocks(int group) { return (group + kCols<T> - 1) / kCols<T>; }

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return bf16_lo(x); }
__device__ __forceinline__ bf16x8 as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8, u); }
__device__ __forceinline__ uint4 load_nt(const char *p) {
  typedef __attribute__((address_space(1))) const u32x4 *global_u32x4;
  const u32x4 w = __builtin_nontemporal_load((global_u32x4)p);
  return make_uint4(w.x, w.y, w.z, w.w);
}
__device__ __forceinline__ int uniform_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
template <typename P>
__device__ __forceinline__ const char *uniform(P x) {     // a wave-uniform address
  const uint64_t a = (uint64_t)x;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return (const char *)((uint64_t)hi << 32 | lo);
}

// Sum of a double over groups of kLanes (4 or 8) lanes; every lane gets it.
template <int kCtrl>
__device__ __forceinline__ double dpp_mov64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, 0xF, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int kLanes>
__device__ __forceinline__ double group_sum(double x) {
  x += dpp_mov64<0xB1>(x);              // lane ^ 1
  x += dpp_mov64<0x4E>(x);              // lane ^ 2
  if (kLanes == 8) x += dpp_mov64<0x141>(x);   // the other half of 8 lanes
  return x;
}

// Reduction over the 4 lane groups (l, l^16, l^32, l^48) of a column.
__device__ __forceinline__ float col_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float col_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// LDS of a workgroup, for at most n blocks of a request, k taken ones and cols columns. The own
// values' way to their operand uses it before, the merge of the waves' states after.
struct Layout {
  uint32_t page, link, sel_k, sel_v, sel_n, extra, bytes;
};
// A wave's own values on their way to the value operand (bf16).
template <typename T, int D>
__host__ __device__ constexpr uint32_t own_scratch() {
  return sizeof(T) == 4 ? 0 : kT * (2 * D + 16);
}
template <typename T, int D>
__host__ __device__ __forceinline__ Layout layout_of(int n, int k, int cols, bool own) {
  Layout l;
  l.page = 8u * n;                      // keys: 8 bytes a block from 0
  l.link = l.page + 4u * n;
  l.sel_k = (l.link + 2u * n + 15) & ~15u;
  l.sel_v = l.sel_k + 8u * k;
  l.sel_n = l.sel_v + 8u * k;
  l.extra = (l.sel_n + 4u * k + 15) & ~15u;
  // fp32: the queries, and each wave's probabilities
  l.bytes = l.extra + (sizeof(T) == 4 ? 4u * kCols<T> * D + 4u * kWaves * kCols<T> * 64 : 0u);
  const uint32_t merge = 4u * kWaves * cols * (D + 2);
  if (l.bytes < merge) l.bytes = merge;
  if (own && l.bytes < own_scratch<T, D>() * kWaves) l.bytes = own_scratch<T, D>() * kWaves;
  return l;
}

// What a unit attends over: the taken blocks (in LDS), then the token's own keys.
struct Unit {
  const uint64_t *k, *v;                // LDS: first K row, V panel of each taken block
  const int32_t *n;                     // LDS: its tokens
  int taken;
  const char *k_own, *v_own;            // the request's first own row, kv head applied
  int64_t own_stride;                   // bytes from own token to own token
  int own;                              // own keys that the token sees
  // log2 of all these keys: the running maxima lie that far above the scores', so that a sum of
  // probabilities is at most one and a sum of values no larger than the largest
  float raise;
};

// ---- bf16 attention: columns of a 16x16x32 product

template <int D>
struct Tile {
  uint4 k[D / 16];                      // 2 key blocks x D / 32 steps
  uint4 v[D / 16];                      // D / 16 value blocks
};
template <int D>
struct State {
  f32x4 o[D / 16];                      // value rows 16 b + 4 (l/16) + i, column l%16
  float m, l;
};

// Tile `half` of a taken block. Key row of M index m of block b: 8 (m/4) + 4 b + m%4, so that
// a lane's scores are the 8 keys of its value operand. Not live: every lane reads the same line.
template <int D>
__device__ __forceinline__ void load_tile(const char *k, const char *v, int half, int lane, bool live,
                                          Tile<D> &x) {
  const int grp = lane >> 4, m = lane & 15;
  const uint32_t mask = live ? ~0u : 0u;
  const uint32_t koff = (uint32_t)(((8 * (m >> 2) + (m & 3)) * D + 8 * grp) * 2) & mask;
  const uint32_t voff = (uint32_t)(m * kT * 2 + 16 * grp) & mask;
  k += half * kT * D * 2;
  v += half * kT * D * 2;
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int s = 0; s < D / 32; ++s) x.k[b * (D / 32) + s] = load_nt(k + koff + (4 * b * D + 32 * s) * 2);
#pragma unroll
  for (int b = 0; b < D / 16; ++b) x.v[b] = load_nt(v + voff + 16 * b * kT * 2);
}
// Own keys j0 .. read in place; keys past `last` reread it (their scores are masked), their
// values are zeros. The values go through LDS (`scratch`, this wave's): gathered from memory two
// bytes at a time, as eight rounds of dependent loads, an own tile held its wave for 16 us in
// a batch that fills HBM.
template <int D>
__device__ __forceinline__ void load_own(const Unit &u, int j0, int last, int lane, char *scratch, Tile<D> &x) {
  constexpr int kRow = 2 * D + 16;      // padded row (bytes)
  const int grp = lane >> 4, m = lane & 15;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const char *row = u.k_own + min(j0 + 8 * (m >> 2) + 4 * b + (m & 3), last) * u.own_stride + 16 * grp;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) x.k[b * (D / 32) + s] = *(const uint4 *)(row + 64 * s);
  }
  uint4 v[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int key = (i * 64 + lane) / (D / 8), c = lane % (D / 8);
    v[i] = *(const uint4 *)(u.v_own + min(j0 + key, last) * u.own_stride + 16 * c);
    if (j0 + key > last) v[i] = make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    *(uint4 *)(scratch + (i * 64 + lane) / (D / 8) * kRow + 16 * (lane % (D / 8))) = v[i];
  __builtin_amdgcn_wave_barrier();
  const char *at = scratch + 8 * grp * kRow + 2 * m;
#pragma unroll
  for (int b = 0; b < D / 16; ++b) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = *(const uint16_t *)(at + 2 * i * kRow + 32 * b) |
             (uint32_t)*(const uint16_t *)(at + (2 * i + 1) * kRow + 32 * b) << 16;
    x.v[b] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __builtin_amdgcn_wave_barrier();
}

// nvalid: keys of the tile that count (may be 0 or less).
template <int D>
__device__ __forceinline__ void compute_tile(const Tile<D> &x, int nvalid, const bf16x8 (&qf)[D / 32],
                                             State<D> &st, int lane, float sc, float raise) {
  f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x.k[s]), qf[s], s0, 0, 0, 0);
    s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x.k[D / 32 + s]), qf[s], s1, 0, 0, 0);
  }
  if (nvalid < kT) {
    const int kl = nvalid - 1 - 8 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i > kl) s0[i] = -INFINITY;
      if (4 + i > kl) s1[i] = -INFINITY;
    }
  }
  float top = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
  top = col_max(top);
  const float mnew = fmaxf(st.m, top * sc + raise);
  if (mnew > st.m) {
    const float alpha = __builtin_amdgcn_exp2f(st.m - mnew);   // 0 when st.m = -inf
    st.l *= alpha;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) st.o[b] *= alpha;
    st.m = mnew;
  }
  const float neg = st.m == -INFINITY ? 0.f : -st.m;
  bf16x8 pf;                            // rounded to bf16 for the value product, 2^-8 of each
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s0[i], sc, neg));
    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1[i], sc, neg));
    pf[i] = (__bf16)p0;
    pf[4 + i] = (__bf16)p1;
    sum += p0 + p1;
  }
  st.l += sum;
#pragma unroll
  for (int b = 0; b < D / 16; ++b)
    st.o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x.v[b]), pf, st.o[b], 0, 0, 0);
}

// A wave's share of a unit: own tiles (before the selection, which they do not wait for), then
// blocks w, w + W, ... of those taken, then its state to LDS (o [cols][D], m and l [cols]).
template <typename T, int D>
struct Attention;

template <int D>
struct Attention<uint16_t, D> {
  bf16x8 qf[D / 32];
  State<D> st;

  __device__ __forceinline__ void start(const uint16_t *q, int cols, int lane, char *) {
    const int col = lane & 15;
    const uint4 *row = (const uint4 *)(q + min(col, cols - 1) * D);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      uint4 x = row[4 * s + (lane >> 4)];
      if (col >= cols) x = make_uint4(0, 0, 0, 0);
      qf[s] = as_bf16x8(x);
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b) st.o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.m = -INFINITY;
    st.l = 0.f;
  }
  __device__ __forceinline__ void own(const Unit &u, int w, int W, int lane, float sc, char *lds) {
    for (int t = W - 1 - w; t * kT < u.own; t += W) {
      Tile<D> x;
      load_own<D>(u, t * kT, u.own - 1, lane, lds + uniform_wave() * own_scratch<uint16_t, D>(), x);
      compute_tile<D>(x, u.own - t * kT, qf, st, lane, sc, u.raise);
    }
  }
  __device__ __forceinline__ void blocks(const Unit &u, int w, int W, int lane, float sc) {
    Tile<D> ta, tb;
    const char *k = nullptr, *v = nullptr;
    int n = 0;
    auto block = [&](int i) {
      k = uniform(u.k[i]);
      v = uniform(u.v[i]);
      n = __builtin_amdgcn_readfirstlane(u.n[i]);
    };
    if (w < u.taken) {
      block(w);
      load_tile<D>(k, v, 0, lane, true, ta);
    }
    // (no branch around the loads: the compiler would wait for all of them where the paths meet)
    for (int i = w; i < u.taken; i += W) {
      load_tile<D>(k, v, 1, lane, n > kT, tb);
      const int n0 = n;
      compute_tile<D>(ta, n0, qf, st, lane, sc, u.raise);
      const bool more = i + W < u.taken;
      if (more) block(i + W);
      load_tile<D>(k, v, 0, lane, more, ta);
      if (n0 > kT) compute_tile<D>(tb, n0 - kT, qf, st, lane, sc, u.raise);
    }
  }
  __device__ __forceinline__ void store(int cols, int lane, float *o, float *m, float *l) {
    const float sum = col_sum(st.l);
    const int col = lane & 15, r4 = 4 * (lane >> 4);
    if (col >= cols) return;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) *(f32x4 *)(o + col * D + 16 * b + r4) = st.o[b];
    if (lane < 16) {
      m[col] = partial_max(st.m, sum);
      l[col] = sum;
    }
  }
};

// fp32 on the vector ALU, up to 4 columns.
template <int D>
struct Attention<float, D> {
  static constexpr int C = 4, E = D / 64;
  const float *qs;                      // LDS: [4][D]
  float *ps;                            // LDS: this wave's probabilities, [4][64]
  float o[C][E], m[C], l[C];

  __device__ __forceinline__ void start(const float *, int, int, char *extra) {
    qs = (const float *)extra;
    ps = (float *)extra + C * D + (threadIdx.x >> 6) * C * 64;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      m[c] = -INFINITY;
      l[c] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[c][e] = 0.f;
    }
  }
  // scores of n keys, a lane one (its row at `row`), and their probabilities to LDS
  __device__ __forceinline__ void scores(const float *row, int n, int lane, float sc, float raise) {
    float s[C] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAhead = 8;           // 16-byte pieces of the row in flight
#pragma unroll 1
    for (int x0 = 0; x0 < D / 4; x0 += kAhead) {
      float4 k4[kAhead];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) k4[x] = ((const float4 *)row)[x0 + x];
#pragma unroll
      for (int x = 0; x < kAhead; ++x)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float4 q4 = ((const float4 *)(qs + c * D))[x0 + x];
          s[c] = __builtin_fmaf(k4[x].x, q4.x, s[c]);
          s[c] = __builtin_fmaf(k4[x].y, q4.y, s[c]);
          s[c] = __builtin_fmaf(k4[x].z, q4.z, s[c]);
          s[c] = __builtin_fmaf(k4[x].w, q4.w, s[c]);
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float x = lane < n ? s[c] * sc : -INFINITY;
      const float mnew = fmaxf(m[c], wave_max(x) + raise);
      const float alpha = mnew == m[c] ? 1.f : __builtin_amdgcn_exp2f(m[c] - mnew);
      const float p = mnew == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - mnew);
      m[c] = mnew;
      l[c] = l[c] * alpha + wave_sum(p);
#pragma unroll
      for (int e = 0; e < E; ++e) o[c][e] *= alpha;
      ps[c * 64 + lane] = p;
    }
    __builtin_amdgcn_wave_barrier();
  }
  __device__ __forceinline__ void own(const Unit &u, int w, int W, int lane, float sc, char *) {
    for (int t = W - 1 - w; t * 64 < u.own; t += W) {
      const int n = min(64, u.own - t * 64);
      scores((const float *)(u.k_own + (t * 64 + min(lane, n - 1)) * u.own_stride), n, lane, sc, u.raise);
#pragma unroll 8
      for (int j = 0; j < n; ++j) {
        const float *v = (const float *)(u.v_own + (int64_t)(t * 64 + j) * u.own_stride);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = v[lane + 64 * e];
#pragma unroll
          for (int c = 0; c < C; ++c) o[c][e] = __builtin_fmaf(ps[c * 64 + j], x, o[c][e]);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  __device__ __forceinline__ void blocks(const Unit &u, int w, int W, int lane, float sc) {
    for (int i = w; i < u.taken; i += W) {
      const char *k = uniform(u.k[i]), *v = uniform(u.v[i]);
      const int n = __builtin_amdgcn_readfirstlane(u.n[i]);
      scores((const float *)k + lane * D, n, lane, sc, u.raise);      // (rows past the last are there, cleared)
#pragma unroll 1
      for (int h = 0; h * kPanel < n; ++h) {                 // panels of 32 tokens
        const float4 *vh = (const float4 *)((const float *)v + (h * D + lane) * kPanel);
        float4 v4[E][kPanel / 4];
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int x = 0; x < kPanel / 4; ++x) v4[e][x] = vh[e * 64 * (kPanel / 4) + x];
#pragma unroll
        for (int x = 0; x < kPanel / 4; ++x)
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const float4 p4 = ((const float4 *)(ps + c * 64 + h * kPanel))[x];
#pragma unroll
            for (int e = 0; e < E; ++e) {
              o[c][e] = __builtin_fmaf(p4.x, v4[e][x].x, o[c][e]);
              o[c][e] = __builtin_fmaf(p4.y, v4[e][x].y, o[c][e]);
              o[c][e] = __builtin_fmaf(p4.z, v4[e][x].z, o[c][e]);
              o[c][e] = __builtin_fmaf(p4.w, v4[e][x].w, o[c][e]);
            }
          }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  __device__ __forceinline__ void store(int cols, int lane, float *o_out, float *m_out, float *l_out) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (c >= cols) break;
#pragma unroll
      for (int e = 0; e < E; ++e) o_out[c * D + lane + 64 * e] = o[c][e];
      if (lane == 0) {
        m_out[c] = partial_max(m[c], l[c]);
        l_out[c] = l[c];
      }
    }
  }
};

// ---- scores and selection

// Scores of n blocks of the unit's request as order-preserving integers in LDS. A lane takes 16
// elements of a summary (with 8, twice as many steps of the sums across lanes: 720 blocks in 13.8
// us, so in 8.7).
template <typename T, int D>
__device__ __forceinline__ void score_blocks(const SparseParams &p, const T *q, int kvh, int n,
                                             const int32_t *page, double *score, int lane, int wave) {
  constexpr int kLanes = D / 16, kRows = 64 / kLanes;    // lanes a summary, summaries a wave
  const int sub = lane % kLanes, rr = lane / kLanes;
  const int64_t row_bytes = (int64_t)p.n_kv_heads * D * 2;
  const char *base = p.means + kvh * D * 2 + sub * 32;
  for (int h0 = 0; h0 < p.group; h0 += 4) {
    double qd[4][16];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) qd[h][i] = (double)to_float(q[min(h0 + h, p.group - 1) * D + sub * 16 + i]);
    constexpr int kAhead = 2;                            // summaries in flight
    for (int b0 = wave * kRows; b0 < n; b0 += kWaves * kRows * kAhead) {
      uint4 c[kAhead][2];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const uint4 *m = (const uint4 *)(base + (int64_t)page[min(b0 + a * kWaves * kRows + rr, n - 1)] * row_bytes);
        c[a][0] = m[0];
        c[a][1] = m[1];
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (b0 + a * kWaves * kRows >= n) break;
        const int b = b0 + a * kWaves * kRows + rr;
        double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 w = c[a][j];
          const double x[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y),
                               bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int h = 0; h < 4; ++h) s[h] = __builtin_fma(qd[h][8 * j + i], x[i], s[h]);
        }
        double best = -INFINITY;                         // (a NaN score counts as -inf)
#pragma unroll
        for (int h = 0; h < 4; ++h) best = fmax(best, group_sum<kLanes>(s[h]));
        if (sub == 0 && b < n) score[b] = h0 == 0 ? best : fmax(best, score[b]);
      }
    }
  }
  __syncthreads();
  uint64_t *key = (uint64_t *)score;
  for (int b = threadIdx.x; b < n; b += kThreads) {
    const uint64_t u = __builtin_bit_cast(uint64_t, score[b] + 0.0);   // (-0 as 0)
    const bool forced = b < p.first || b >= n - p.last;
    key[b] = forced ? ~0ull : u >> 63 ? ~u : u | 1ull << 63;
  }
  __syncthreads();
}

// Lists the `take` (below n) blocks of the largest keys, ascending: list(at, block). (Each thread
// counting the keys before its block's, for few blocks: 170 blocks 3.5 us, 256 5.7; so 3.2, 3.4.)
template <typename F>
__device__ __forceinline__ void select_blocks(const uint64_t *key, int n, int take, F list) {
  __shared__ uint32_t hist[256], found[3], part[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t at = 0, mask = 0;            // the smallest key taken, as far as it is known
  int need = take;                      // of those that agree with it so far
  bool whole = false;                   // all of them are taken
  for (int shift = 56; shift >= 0 && !whole; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int b = tid; b < n; b += kThreads)
      if (((key[b] ^ at) & mask) == 0) atomicAdd(&hist[(key[b] >> shift) & 255], 1u);
    __syncthreads();
    if (wave == 0) {                    // a lane 4 bins, from the largest
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += c[i] = hist[255 - 4 * lane - i];
      uint32_t upto = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o);
        if (lane >= o) upto += x;
      }
      uint32_t above = upto - sum;
      if (above < (uint32_t)need && (uint32_t)need <= upto) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < (uint32_t)need && (uint32_t)need <= above + c[i]) {
            found[0] = 255 - 4 * lane - i;
            found[1] = above;
            found[2] = c[i];
          }
          above += c[i];
        }
      }
    }
    __syncthreads();
    at |= (uint64_t)found[0] << shift;
    mask |= 255ull << shift;
    need -= (int)found[1];
    whole = (int)found[2] == need;
  }
  // larger ones and, of the equal ones, the first `need`; a thread a range of blocks
  const int per = (n + kThreads - 1) / kThreads, b0 = min(n, tid * per), b1 = min(n, b0 + per);
  uint32_t mine = 0;                    // counts: larger | equal << 16
  for (int b = b0; b < b1; ++b) {
    const uint64_t x = key[b] & mask;
    mine += x > at ? 1u : x == at ? 1u << 16 : 0u;
  }
  uint32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  uint32_t before = upto - mine;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) before += w < wave ? part[w] : 0u;
  int more = before & 0xffff, equal = before >> 16;
  for (int b = b0; b < b1; ++b) {
    const uint64_t x = key[b] & mask;
    if (x > at) {
      list(more + min(equal, need), b);
      ++more;
    } else if (x == at) {
      if (equal < need) list(more + equal, b);
      ++equal;
    }
  }
  __syncthreads();
}

template <typename T, int D>
__device__ __forceinline__ void link_sparse(const SparseParams &p, const SparseLink *links,
                                            const SparseToken *tokens) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, wave = uniform_wave();
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  const int cb = x % p.col_blocks;
  x /= p.col_blocks;
  const int kvh = x % p.n_kv_heads, tok = p.token0 + x / p.n_kv_heads;
  const SparseToken R = tokens[tok];
  const int n = R.blocks, take = min(n, p.n_blocks);
  const Layout at = layout_of<T, D>(p.most_blocks, p.n_blocks, p.cols, p.k_self != nullptr);
  int32_t *page = (int32_t *)(lds + at.page);
  uint16_t *link = (uint16_t *)(lds + at.link);
  uint64_t *sel_k = (uint64_t *)(lds + at.sel_k), *sel_v = (uint64_t *)(lds + at.sel_v);
  int32_t *sel_n = (int32_t *)(lds + at.sel_n);
  const T *q = (const T *)p.q + ((int64_t)tok * p.n_q_heads + kvh * p.group) * D;

  const int col0 = cb * kCols<T>, cols = min(kCols<T>, p.group - col0);
  // (the first blocks go to the first wave of every split, which has a SIMD to itself)
  const int w = wave * p.splits + split, W = p.splits * kWaves;
  Unit u;
  u.k = sel_k;
  u.v = sel_v;
  u.n = sel_n;
  u.taken = take;
  u.own_stride = (int64_t)p.n_kv_heads * D * (int)sizeof(T);
  const int64_t own_at = R.s0 * u.own_stride + kvh * D * (int)sizeof(T);
  u.k_own = (const char *)p.k_self + own_at;
  u.v_own = (const char *)p.v_self + own_at;
  u.own = R.own;
  // (whole powers of two: the probability of a score at the maximum stays exact in bf16; error of
  // a batch's outputs 2.0e-3, else 2.3e-3)
  u.raise = ceilf(log2f((float)(take * kTile + R.own + 1)));
  Attention<T, D> att;
  att.start(q + col0 * D, cols, lane, lds + at.extra);
  if (sizeof(T) == 4) {
    for (int i = threadIdx.x; i < kCols<T> * D; i += kThreads)
      ((float *)(lds + at.extra))[i] = i < cols * D ? to_float(q[col0 * D + i]) : 0.f;
    __syncthreads();
  }
  // (the first round of links is on its way under the own tiles)
  links += R.link0;
  struct Span {
    int tile0, page, tiles;
  };
  auto span = [&](int l0) {
    const int l = l0 + lane * kWaves + wave;
    const SparseLink *L = links + min(l, R.nlinks - 1);
    return Span{L->tile0, L->page, l < R.nlinks ? (L->len + kTile - 1) / kTile : 0};
  };
  Span sp = R.nlinks > 0 ? span(0) : Span{0, 0, 0};
  att.own(u, w, W, lane, p.scale_log2, lds);
  if (sizeof(T) == 2 && u.own > 0) __syncthreads();

  // every block's page and link: a wave loads 64 links at once, then walks them
  for (int l0 = 0; l0 < R.nlinks; l0 += 64 * kWaves) {
    if (l0 > 0) sp = span(l0);
    for (int i = 0; i < 64 && l0 + i * kWaves + wave < R.nlinks; ++i) {
      const int t0 = __builtin_amdgcn_readlane(sp.tile0, i), p0 = __builtin_amdgcn_readlane(sp.page, i);
      const int nt = __builtin_amdgcn_readlane(sp.tiles, i);
      for (int t = lane; t < nt; t += 64) {
        page[t0 + t] = p0 + t;
        link[t0 + t] = (uint16_t)(l0 + i * kWaves + wave);
      }
    }
  }
  __syncthreads();

  int32_t *taken = p.taken && cb == 0 && split == 0 ? p.taken + ((int64_t)tok * p.n_kv_heads + kvh) * p.n_blocks : nullptr;
  auto list = [&](int i, int b) {
    const SparseLink L = links[link[b]];
    const int64_t t = (int64_t)(b - L.tile0) * kTile;
    sel_k[i] = (uint64_t)(L.k + ((int64_t)kvh * L.lp + t) * D * (int)sizeof(T));
    sel_v[i] = (uint64_t)(L.v + ((int64_t)kvh * D * L.lp + t * D) * (int)sizeof(T));
    sel_n[i] = min(kTile, L.len - (int)t);
    if (taken) taken[i] = b;
  };
  if (take == n) {                      // all of them
    for (int b = threadIdx.x; b < n; b += kThreads) list(b, b);
  } else {
    score_blocks<T, D>(p, q, kvh, n, page, (double *)lds, lane, wave);
    select_blocks((const uint64_t *)lds, n, take, list);
  }
  if (taken)
    for (int i = take + (int)threadIdx.x; i < p.n_blocks; i += kThreads) taken[i] = -1;

  __syncthreads();
  att.blocks(u, w, W, lane, p.scale_log2);
  __syncthreads();                      // the lists are done with
  const int stride = p.cols;            // columns of a wave's state
  float *o = (float *)lds, *m = o + kWaves * stride * D, *l = m + kWaves * stride;
  att.store(cols, lane, o + wave * stride * D, m + wave * stride, l + wave * stride);
  __syncthreads();

  // the waves' states merged: a thread 4 dims of a column
  for (int i = threadIdx.x; i < cols * (D / 4); i += kThreads) {
    const int c = i / (D / 4), e = (i - c * (D / 4)) * 4;
    float M = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, m[w * stride + c]);
    float f[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      f[w] = m[w * stride + c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[w * stride + c] - M);
      sum += f[w] * l[w * stride + c];
    }
    // (normalised here with weights that sum to one: sums of large values stay finite)
    const float inv = p.splits > 1 ? 1.f : sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (f[w] == 0.f) continue;
      const float4 v = *(const float4 *)(o + (w * stride + c) * D + e);
      const float g = f[w] * inv;
      a = make_float4(a.x + g * v.x, a.y + g * v.y, a.z + g * v.z, a.w + g * v.w);
    }
    const int64_t row = (int64_t)tok * p.n_q_heads + kvh * p.group + col0 + c;
    if (p.splits > 1) {
      const int64_t pr = (int64_t)split * p.total_q * p.n_q_heads + row;
      *(float4 *)(p.part.o + pr * D + e) = a;
      if (e == 0) {
        p.part.m[pr] = M;
        p.part.l[pr] = sum;
      }
      continue;
    }
    if (sizeof(T) == 4) {
      *(float4 *)((float *)p.out + row * D + e) = a;
    } else {
      const __bf16 r[4] = {(__bf16)a.x, (__bf16)a.y, (__bf16)a.z, (__bf16)a.w};
      *(uint2 *)((uint16_t *)p.out + row * D + e) = __builtin_bit_cast(uint2, r);
    }
    if (p.lse && e == 0) p.lse[row] = M == -INFINITY ? -INFINITY : log_sum(M, sum);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 1) void link_sparse_kernel(SparseParams p) {
  link_sparse<T, D>(p, p.links, p.tokens);
}
// Tables of a small call as a kernel argument.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, 1) void link_sparse_tabs_kernel(SparseParams p, SparseTabs t) {
  link_sparse<T, D>(p, t.links, t.tokens);
}

template <typename T, int D>
hipError_t launch_sparse_t(SparseParams p, const SparseTabs *tabs, hipStream_t st) {
  p.col_blocks = col_blocks<T>(p.group);
  p.cols = std::min(kCols<T>, p.group);
  const size_t lds = layout_of<T, D>(p.most_blocks, p.n_blocks, p.cols, p.k_self != nullptr).bytes;
  const void *f = tabs ? (const void *)link_sparse_tabs_kernel<T, D> : (const void *)link_sparse_kernel<T, D>;
  hipError_t e = hipSuccess;
  if (lds > 64 * 1024) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  // (a launch's threads are counted in 32 bits)
  const int64_t per = (int64_t)p.n_kv_heads * p.col_blocks * p.splits;
  const int64_t most = std::max<int64_t>(1, ((1 << 23) - 1) / per);
  for (int64_t at = 0; at < p.total_q; at += most) {
    p.token0 = (int32_t)at;
    const dim3 grid((unsigned)(std::min<int64_t>(most, p.total_q - at) * per));
    if (tabs)
      hipLaunchKernelGGL((link_sparse_tabs_kernel<T, D>), grid, dim3(kThreads), lds, st, p, *tabs);
    else
      hipLaunchKernelGGL((link_sparse_kernel<T, D>), grid, dim3(kThreads), lds, st, p);
  }
  return hipGetLastError();
}

// Means of the pages of a run: page blockIdx.x, head and piece blockIdx.y, layer blockIdx.z.
// Bound by the keys' bytes, read once: 96 chunks of 1024 tokens, 8 heads x 128 bf16, 33.8 us (201 MB, 6.0
// TB/s), in 8 layers 296 (5.4), one of 60,000 tokens 19 (6.4); a grown page of each of 64 chunks 3.6 us.
// Every piece gets the workgroups of the launch's longest: that one of 60,000 tokens and 95 of 64
// in one call take 169 us. Sums in 64 bits (those of 64 bf16 numbers are exact over
// 40 binary orders), the mean rounded to fp32 and then to bf16.
template <typename T, int D>
__global__ __launch_bounds__(256) void block_means_kernel(MeansParams p) {
  constexpr int kParts = 256 / D;
  __shared__ double sums[256];
  const int h = blockIdx.y % p.heads;
  const MeansPiece P = p.piece[blockIdx.y / p.heads];
  const int e = threadIdx.x % D, part = threadIdx.x / D;
  for (int pg = blockIdx.x; pg * kTile < P.n; pg += gridDim.x) {
    const int rows = min(kTile, P.n - pg * kTile);
    const T *k = (const T *)(P.k + blockIdx.z * p.layer_bytes) + ((int64_t)h * P.lp + pg * kTile) * D + e;
    double s = 0.0;
#pragma unroll 8
    for (int r = part; r < rows; r += kParts) s += (double)to_float(k[r * D]);
    sums[threadIdx.x] = s;
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int i = 1; i < kParts; ++i) s += sums[i * D + e];
      ((__bf16 *)p.means)[blockIdx.z * p.layer_elems + ((int64_t)(P.page + pg) * p.heads + h) * D + e] =
          (__bf16)(float)(s / rows);
    }
    __syncthreads();
  }
}

}  // namespace

bool sparse_supported(int dtype, int mla, int d_k, int d_v) {
  return !mla && d_k == d_v && (d_k == 64 || d_k == 128) && (dtype == 0 || dtype == 1);
}

int sparse_columns(int dtype, int group) { return dtype == 0 ? col_blocks<float>(group) : col_blocks<uint16_t>(group); }

hipError_t launch_link_sparse(const SparseParams &p, const SparseTabs *tabs, int dtype, int d, hipStream_t st) {
  if (dtype == 0)
    return d == 64 ? launch_sparse_t<float, 64>(p, tabs, st) : launch_sparse_t<float, 128>(p, tabs, st);
  return d == 64 ? launch_sparse_t<uint16_t, 64>(p, tabs, st) : launch_sparse_t<uint16_t, 128>(p, tabs, st);
}

hipError_t launch_block_means(const MeansParams &p, int32_t n, int32_t n_layers, int dtype, int d, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  int most = 1;
  for (int i = 0; i < n; ++i) most = std::max(most, (p.piece[i].n + kTile - 1) / kTile);
  const dim3 grid((unsigned)std::min(most, 4096), (unsigned)(n * p.heads), (unsigned)n_layers);
  if (dtype == 0) {
    if (d == 64)
      hipLaunchKernelGGL((block_means_kernel<float, 64>), grid, dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL((block_means_kernel<float, 128>), grid, dim3(256), 0, st, p);
  } else {
    if (d == 64)
      hipLaunchKernelGGL((block_means_kernel<uint16_t, 64>), grid, dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL((block_means_kernel<uint16_t, 128>), grid, dim3(256), 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace pic
