// Link attention over a 4-bit chunk cache on gfx950 for calls with few rows per kv
// head: a workgroup takes 16 or 32 rows (query token x query head) of one kv head over a
// piece of a request's keys, each of its four waves every fourth 64-key tile of it. (32
// rows where a request has more than 16: keys and values are widened once for both
// blocks of 16.)
//
// At the end the waves' states become one through LDS, and only then a partial is
// written, or the output itself: with one wave per piece, four times as many partials
// were written and combined (one request of 37 tokens over 112 tiles 26.2 -> 20.2 us, of
// 16 tokens 18.9 -> 13.4; 64 decode requests over 8 shared documents, now in one piece, 76
// -> 59; 64-wide heads, 37 tokens, 21.8 -> 14.0).
//
// Bound by the cache's bytes where a batch fills the GPU: 64 decode requests over 16
// links of 1024 and 128 own tokens, 32/8 heads x 128, 1.18 GB in 171 us, 6.9 TB/s of
// the 7.1 of a plain read stream. Else by the latency of a wave's tiles, about 1.2 us
// each, between some 3 us of start (tables, queries, first tile) and end.
//
// The tiles of the cache hold their codes in the order of the matrix
// operands (fp4.hpp), so a wave streams them from HBM into registers, 1 KB per
// load, widens them there (a conversion that takes the block's scale: one
// instruction per two elements) and multiplies:
//   S^T[64 keys][16 rows] = K . Q^T       4 key blocks x D/32 steps of
//                                         v_mfma_f32_16x16x32_bf16
//   O^T[D][16 rows]      += V^T . P^T     D/16 channel blocks x 2 steps
// After the first product lane (n, g) holds the scores of row n for the keys
// 16 b + 4 g + i, which are the keys that its operand of the second one
// needs: no exchange between lanes. Value codes lie key by key with their channels
// side by side (a row has its own scales); conversions give pairs of
// channels, and one byte permute per pair of keys turns them into pairs of keys.
// Channel block cb, index m is channel D/16 * m + cb, so that a lane ends with
// D/16 neighbouring channels.
//
// The own KV is bf16 and read in place, 32 keys at a time, its key rows as they
// are and its value rows through the same permutes.
//
// Softmax: log2 domain, exact running max per tile, sums of the probabilities
// in fp32 before they are rounded to bf16 for the matrix product (half a step, at
// most 2^-8 of each, as wide as the output's own rounding; keys and values are exact
// in bf16). The scaled matrix instructions would take the codes as they are, with
// the query as a sum of two 8-bit numbers, at the same rate; their inner sums keep
// fewer bits (scores of size 11 were off by up to 4.8e-4, these by 1.9e-6).
#include "fp4.hpp"

namespace pic {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const u32x4 *global_u32x4;

constexpr int kWaves = 4;

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8, u); }
__device__ __forceinline__ uint32_t word(uint4 u, int i) {
  return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
}

// Reduction over the 4 lane groups (l, l^16, l^32, l^48) of a row.
__device__ __forceinline__ float row_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <bool kOnce>
__device__ __forceinline__ uint4 load_codes(const char *p) {
  const u32x4 w = kOnce ? __builtin_nontemporal_load((global_u32x4)p) : *(global_u32x4)p;
  return make_uint4(w.x, w.y, w.z, w.w);
}

// A 64-key tile of the cache as loaded. kOnce: its codes pass the caches by. Chosen by the
// rows of a request alone: those of one row block (up to 16 rows), whose documents may be its
// own (64 decode requests with 16 of their own each, 1 GB: 177 us, cached 207; 64-wide heads
// 93, 108). Where several row blocks read them, cached is faster (16 requests of 16 tokens
// over 4..12 of 64 documents, 51 -> 47 us, 64-wide 38 -> 34). Documents that decode requests
// share would rather be cached, too, from about two readers each on: 64 requests over 16 of
// 1024 documents 167 us, cached 169 (64-wide 92, 88), of 64 documents 138, 114 (85, 75), over
// 8 of 8 67, 64 (43, 42), 16 requests of 1..4 tokens over 4..12 of 64 20.3, 20.3 (14.4, 14.0).
template <int D, bool kOnce>
struct CacheTile {
  static constexpr int kKeyBlocks = 4;
  uint4 k[D / 32], v[D / 32];
  uint32_t ks;      // K scales of key blocks 0..3 (this lane's block of 32)
  uint4 vs;         // V scales of keys 16 b + 4 g + i (this lane's channels)

  __device__ __forceinline__ void load(const char *tile, int lane) {
    typedef Fp4Tile<D> T;
    const int m = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      k[j] = load_codes<kOnce>(tile + j * 1024 + lane * 16);
      v[j] = load_codes<kOnce>(tile + T::kV + j * 1024 + lane * 16);
    }
    const int kc = D == 128 ? g : g >> 1;
    const int vc = m * (D / 16) / 32;
    ks = *(const uint32_t *)(tile + T::kKs + (kc * 16 + m) * 4);
    vs = *(const uint4 *)(tile + T::kVs + (g * T::kBlocks + vc) * 16);
  }
  // Operand of key block b, step s: elements D/4 * g + 8 s ..+7 of key 16 b + m.
  __device__ __forceinline__ bf16x8 key(int b, int s) const {
    const float sc = fp4_scale((ks >> (8 * b)) & 255u);
    const uint32_t c = D == 128 ? word(k[b % (D / 32)], s)
                                : word(k[b / 2 % (D / 32)], 2 * (b & 1) + s);
    return as_bf16x8(fp4_decode8(c, sc));
  }
  // Channels 2 c, 2 c + 1 of this lane's, key 16 b + 4 g + i.
  template <int kC>
  __device__ __forceinline__ uint32_t value(int b, int i) const {
    const float sc = fp4_scale((word(vs, b) >> (8 * i)) & 255u);
    if constexpr (D == 128) {
      return fp4_pair<kC>(word(v[b % (D / 32)], i), sc);
    } else {
      const uint32_t w = word(v[b / 2 % (D / 32)], 2 * (b & 1) + (i >> 1));
      return (i & 1) ? fp4_pair<2 + (kC & 1)>(w, sc) : fp4_pair<kC & 1>(w, sc);
    }
  }
};

// 32 own keys, read in place. k, v: this kv head's first own row; stride: bytes per
// token. Keys past the last own one reread it (their scores are masked), with
// zeros for values: 0 times an infinity would be a NaN.
template <int D>
struct OwnTile {
  static constexpr int kKeyBlocks = 2;
  uint4 k[2][D / 32];
  uint32_t v[2][4][D / 32];

  __device__ __forceinline__ void load(const char *kr, const char *vr, int64_t stride, int j0,
                                       int last, int lane) {
    const int m = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char *row = kr + min(j0 + 16 * b + m, last) * stride + g * (D / 2);
#pragma unroll
      for (int s = 0; s < D / 32; ++s) k[b][s] = *(const uint4 *)(row + 16 * s);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = j0 + 16 * b + 4 * g + i;
        const char *vp = vr + min(key, last) * stride + m * (D / 8);
        const uint32_t keep = key <= last ? ~0u : 0u;
#pragma unroll
        for (int c = 0; c < D / 32; c += 2) {
          const uint2 w = *(const uint2 *)(vp + 4 * c);
          v[b][i][c] = w.x & keep;
          v[b][i][c + 1] = w.y & keep;
        }
      }
    }
  }
  __device__ __forceinline__ bf16x8 key(int b, int s) const { return as_bf16x8(k[b][s]); }
  template <int kC>
  __device__ __forceinline__ uint32_t value(int b, int i) const {
    return v[b][i][kC];
  }
};

// NB: blocks of 16 rows that a wave takes.
template <int D, int NB>
struct State {
  f32x4 o[NB][D / 16];   // channel block cb: channels D/16 * (4 g + i) + cb of row n
  float m[NB], l[NB];    // running max (log2 domain, per row) and this lane's part of the sum
};

template <int D, int NB, int kC, class Tile>
__device__ __forceinline__ void value_pair(const Tile &x, int t, const bf16x8 (&pf)[NB],
                                           State<D, NB> &st) {
  uint32_t d[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d[i] = x.template value<kC>(2 * t, i);
    d[4 + i] = x.template value<kC>(2 * t + 1, i);
  }
  const uint4 lo = make_uint4(__builtin_amdgcn_perm(d[1], d[0], 0x05040100u),
                              __builtin_amdgcn_perm(d[3], d[2], 0x05040100u),
                              __builtin_amdgcn_perm(d[5], d[4], 0x05040100u),
                              __builtin_amdgcn_perm(d[7], d[6], 0x05040100u));
  const uint4 hi = make_uint4(__builtin_amdgcn_perm(d[1], d[0], 0x07060302u),
                              __builtin_amdgcn_perm(d[3], d[2], 0x07060302u),
                              __builtin_amdgcn_perm(d[5], d[4], 0x07060302u),
                              __builtin_amdgcn_perm(d[7], d[6], 0x07060302u));
#pragma unroll
  for (int r = 0; r < NB; ++r) {
    st.o[r][2 * kC] =
        __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(lo), pf[r], st.o[r][2 * kC], 0, 0, 0);
    st.o[r][2 * kC + 1] =
        __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(hi), pf[r], st.o[r][2 * kC + 1], 0, 0, 0);
  }
}

// kl: last visible key of the tile for this lane's rows (relative to the tile),
// used where masked. bias: added to its maximum.
template <int D, int NB, class Tile>
__device__ __forceinline__ void compute_tile(const Tile &x, const bf16x8 (&qf)[NB][D / 32],
                                             State<D, NB> &st, int lane, bool masked,
                                             const int (&kl)[NB], float sc, float bias) {
  constexpr int kB = Tile::kKeyBlocks;
  f32x4 s[NB][kB];
#pragma unroll
  for (int b = 0; b < kB; ++b) {
#pragma unroll
    for (int r = 0; r < NB; ++r) s[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const bf16x8 k = x.key(b, j);
#pragma unroll
      for (int r = 0; r < NB; ++r)
        s[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[r][j], s[r][b], 0, 0, 0);
    }
  }
  if (masked) {
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      const int k0 = kl[r] - 4 * (lane >> 4);
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * b + i > k0) s[r][b][i] = -INFINITY;
    }
  }
  float neg_m[NB];
#pragma unroll
  for (int r = 0; r < NB; ++r) {
    float tmax = -INFINITY;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) tmax = fmaxf(tmax, s[r][b][i]);
    tmax = row_max(tmax);
    const float mnew = fmaxf(st.m[r], __builtin_fmaf(tmax, sc, bias));
    if (mnew > st.m[r]) {        // per lane: rescale this row's state
      const float alpha = __builtin_amdgcn_exp2f(st.m[r] - mnew);   // 0 when m = -inf
      st.l[r] *= alpha;
#pragma unroll
      for (int b = 0; b < D / 16; ++b) st.o[r][b] *= alpha;
      st.m[r] = mnew;
    }
    neg_m[r] = st.m[r] == -INFINITY ? 0.f : -st.m[r];
  }
#pragma unroll
  for (int t = 0; t < kB / 2; ++t) {
    bf16x8 pf[NB];
#pragma unroll
    for (int r = 0; r < NB; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][2 * t][i], sc, neg_m[r]));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][2 * t + 1][i], sc, neg_m[r]));
        st.l[r] += p0 + p1;
        pf[r][i] = (__bf16)p0;
        pf[r][4 + i] = (__bf16)p1;
      }
    value_pair<D, NB, 0>(x, t, pf, st);
    value_pair<D, NB, 1>(x, t, pf, st);
    if constexpr (D == 128) {
      value_pair<D, NB, 2>(x, t, pf, st);
      value_pair<D, NB, 3>(x, t, pf, st);
    }
  }
}

// LDS of the merge: per wave and row its output (rows 4 floats apart beyond their
// length, so that 16 rows' chunks lie in different banks), maximum and sum.
template <int D, int NB>
struct Merge {
  static constexpr int kRows = 16 * NB, kStride = D + 4;
  static constexpr int kMax = kWaves * kRows * kStride, kSum = kMax + kWaves * kRows;
  static constexpr int kFlag = kSum + kWaves * kRows;    // per wave: its sums are too large
  static constexpr int kFloats = kFlag + kWaves;
};

// Largest sum that the merge adds four of without leaving the fp32 range.
constexpr float kSafeSum = 0x1p125f;

struct TileInfo {
  const char *p;
  int nvalid, tok;
};

// kLim: rows see different numbers of linked rows. big: the second pass (see fp4_bias). Returns
// whether the workgroup's sums came out too large in the first one (and nothing was written).
template <int D, bool kLim, int NB, bool kArg>
__device__ __forceinline__ bool link_body(int wave, bool big) {
  const Fp4Start<kArg> start(wave);
  const LinkParams &p = start.p;
  typedef Merge<D, NB> M;
  __shared__ __align__(16) float lds[M::kFloats];
  const int lane = start.lane;
  // Row blocks of a unit (item, kv head) are neighbours on one XCD: they read the same
  // tiles at about the same time. (In the order of the launch: 20.2 -> 18.6 us for one
  // request of 37 tokens, 189 -> 182 for 32 of 16 over 16 documents of their own.)
  const UnitBlock ub = unit_of_block(start.block, p.nrb, p.n_xcd, 0, p.n_items * p.n_kv_heads);
  const int u = ub.u, rb = ub.rb;
  if (u >= p.n_items * p.n_kv_heads) return false;
  const int kvh = u % p.n_kv_heads;
  const WorkItem it = load_item(start.items, u / p.n_kv_heads);
  const ReqEntry R = item_request(it);
  const int group = p.group;
  const int nrows = R.lq * group, row0 = rb * (16 * NB);
  if (row0 >= nrows) return false;

  // this lane's rows
  const int n = lane & 15, g = lane >> 4;
  bool rvalid[NB];
  int own_last[NB], dl[NB], dmin = kNoLimit, dmax = 0;                // own_last: last visible own key
  int64_t orow[NB];
#pragma unroll
  for (int r = 0; r < NB; ++r) {
    const int row = row0 + 16 * r + n;
    rvalid[r] = row < nrows;
    const int qi = rvalid[r] ? row / group : 0;
    own_last[r] = rvalid[r] ? qi + R.ls - R.lq : -1;
    orow[r] = (int64_t)(R.q0 + qi) * p.n_q_heads + kvh * group + (rvalid[r] ? row % group : 0);
    dl[r] = kNoLimit;
    if (kLim) {
      if (rvalid[r]) dl[r] = p.doc_lim[R.q0 + qi];
      dmin = min(dmin, dl[r]);
      dmax = max(dmax, rvalid[r] ? dl[r] : 0);
    }
  }
  if (kLim) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      dmin = min(dmin, __shfl_xor(dmin, o));
      dmax = max(dmax, __shfl_xor(dmax, o));
    }
    dmin = __builtin_amdgcn_readfirstlane(dmin);
    dmax = __builtin_amdgcn_readfirstlane(dmax);
  }

  LinkCursor<true> c;
  c.start(start.links, it);
  auto info = [&](int t) {       // t only grows
    while (t >= c.end) c.next();
    const int tt = t - c.tile0;
    return TileInfo{c.base + ((int64_t)tt * p.n_kv_heads + kvh) * Fp4Tile<D>::kBytes,
                    min(kTile, c.len - tt * kTile), c.tok0 + tt * kTile};
  };
  // this wave's tiles: every fourth
  const int t_first = it.t_begin + wave, doc_end = min(it.t_end, R.doc_tiles);
  CacheTile<D, NB == 1> ta, tb;
  TileInfo ia{}, ib{};
  if (t_first < doc_end) {
    ia = info(t_first);
    ta.load(ia.p, lane);
  }
  bf16x8 qf[NB][D / 32];
  State<D, NB> st;
#pragma unroll
  for (int r = 0; r < NB; ++r) {
    const uint4 *qrow = (const uint4 *)((const uint16_t *)p.q + orow[r] * D + g * (D / 4));
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (rvalid[r]) v = qrow[s];
      qf[r][s] = as_bf16x8(v);
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b) st.o[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.m[r] = -INFINITY;
    st.l[r] = 0.f;
  }
  const float sc = p.scale_log2;
  const float bias = big ? fp4_bias(max(1, it.t_end - it.t_begin)) : 0.f;
  auto doc_tile = [&](const CacheTile<D, NB == 1> &x, const TileInfo &i) {
    const bool masked = i.nvalid < kTile || (kLim && i.tok + kTile > dmin);
    int kl[NB];
#pragma unroll
    for (int r = 0; r < NB; ++r) kl[r] = (kLim ? min(i.nvalid, dl[r] - i.tok) : i.nvalid) - 1;
    compute_tile<D, NB>(x, qf, st, lane, masked, kl, sc, bias);
  };
  // The load past the last tile reads the piece's last one, which keeps the
  // loop free of branches around loads (the compiler waits for every load in
  // flight where such paths meet). It ends where no row sees a linked one any more.
  for (int t = t_first; t < doc_end; t += 2 * kWaves) {
    if (kLim && ia.tok >= dmax) break;
    ib = info(min(t + kWaves, doc_end - 1));
    tb.load(ib.p, lane);
    doc_tile(ta, ia);
    if (t + kWaves >= doc_end || (kLim && ib.tok >= dmax)) break;
    ia = info(min(t + 2 * kWaves, doc_end - 1));
    ta.load(ia.p, lane);
    doc_tile(tb, ib);
  }
  // Own tiles up to the one that holds the block's last visible key.
  const int last_qi = (min(row0 + 16 * NB, nrows) - 1) / group;
  const int t_end = min(it.t_end, visible_tiles(R, last_qi));
  int own = max(it.t_begin, R.doc_tiles);
  own += (t_first - own) & (kWaves - 1);
  if (own < t_end) {
    int s0 = it.tok0;             // the own link's: its first own row
    if (it.tile0 < R.doc_tiles) {
      while (c.tile0 < R.doc_tiles) c.next();
      s0 = c.tok0;
    }
    const int64_t at = ((int64_t)s0 * p.n_kv_heads + kvh) * D * 2;
    const int64_t stride = (int64_t)p.n_kv_heads * D * 2;
    for (; own < t_end; own += kWaves) {
      const int k0 = (own - R.doc_tiles) * kTile, k_end = min(R.ls, k0 + kTile);
      for (int j0 = k0; j0 < k_end; j0 += 32) {
        OwnTile<D> x;
        x.load((const char *)p.k_self + at, (const char *)p.v_self + at, stride, j0, R.ls - 1, lane);
        int kl[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) kl[r] = min(own_last[r], R.ls - 1) - j0;
        compute_tile<D, NB>(x, qf, st, lane, true, kl, sc, bias);
      }
    }
  }

  // The waves' states of each row become one: its largest maximum M, sums and outputs
  // times 2^(m - M), added in the order of the waves.
  float *const mb = lds + M::kMax, *const lb = lds + M::kSum;
#pragma unroll
  for (int r = 0; r < NB; ++r) {
    const float ltot = row_sum(st.l[r]);
    st.m[r] = partial_max(st.m[r], ltot);
    if (g == 0) {
      mb[wave * M::kRows + 16 * r + n] = st.m[r];
      lb[wave * M::kRows + 16 * r + n] = ltot;
    }
  }
  if (!big) {       // (not in the second pass: another wave may still read the first one's flags)
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < NB; ++r)
#pragma unroll
      for (int b = 0; b < D / 16; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = __builtin_elementwise_maximum(most, fabsf(st.o[r][b][i]));
    const bool over = __any(!(most <= kSafeSum));
    if (lane == 0) lds[M::kFlag + wave] = over ? 1.f : 0.f;
  }
  __syncthreads();
  if (!big) {
    float over = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) over += lds[M::kFlag + w];
    if (__builtin_expect(over != 0.f, 0)) return true;
  }
#pragma unroll
  for (int r = 0; r < NB; ++r) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, mb[w * M::kRows + 16 * r + n]);
    const float f = __builtin_amdgcn_exp2f(st.m[r] - top);
    float *row = lds + (wave * M::kRows + 16 * r + n) * M::kStride + D / 4 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int b = 0; b < D / 16; b += 4) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);      // (a wave that saw no key: not times 0)
        if (st.m[r] != -INFINITY)
          v = make_float4(st.o[r][b][i] * f, st.o[r][b + 1][i] * f, st.o[r][b + 2][i] * f,
                          st.o[r][b + 3][i] * f);
        *(float4 *)(row + D / 16 * i + b) = v;
      }
  }
  __syncthreads();
  // four channels of a row per thread and step
  for (int e = 64 * wave + lane; e < M::kRows * (D / 4); e += 64 * kWaves) {
    const int row = e / (D / 4), ch = e % (D / 4) * 4;
    if (row0 + row >= nrows) break;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, mb[w * M::kRows + row]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float m = mb[w * M::kRows + row];
      if (m != -INFINITY) sum += lb[w * M::kRows + row] * __builtin_amdgcn_exp2f(m - top);
      const float4 x = *(const float4 *)(lds + (w * M::kRows + row) * M::kStride + ch);
      o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
    }
    const int q = (row0 + row) / group;
    const int64_t in_req = (int64_t)q * p.n_q_heads + kvh * group + (row0 + row) % group;
    const int64_t to = (int64_t)R.q0 * p.n_q_heads + in_req;
    if (it.part < 0) {
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      bf16x4v v;
      v[0] = (__bf16)(o.x * inv), v[1] = (__bf16)(o.y * inv);
      v[2] = (__bf16)(o.z * inv), v[3] = (__bf16)(o.w * inv);
      *(uint2 *)((uint16_t *)p.out + to * D + ch) = __builtin_bit_cast(uint2, v);
      if (p.lse && ch == 0) p.lse[to] = sum == 0.f ? -INFINITY : log_sum(top, sum);
    } else {
      const int64_t prow = it.part + in_req;
      *(float4 *)(p.part_o + prow * D + ch) = o;
      if (ch == 0) {
        p.part_m[prow] = partial_max(top, sum);
        p.part_l[prow] = sum;
      }
    }
  }
  return false;
}

template <int D, bool kLim, int NB, bool kArg>
__device__ __forceinline__ void link_piece() {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (bool big = false; link_body<D, kLim, NB, kArg>(wave, big); big = true) {
  }
}

template <int D, bool kLim, int NB>
__global__ __launch_bounds__(256, 2) void link_fp4_kernel(LinkParams) {
  link_piece<D, kLim, NB, false>();
}

// The tables are read where they are, in the kernel arguments.
template <int D, int NB>
__global__ __launch_bounds__(256, 2) void link_fp4_tabs_kernel(Fp4Args) {
  link_piece<D, false, NB, true>();
}

template <int D, int NB>
void launch(const LinkParams &p, const Fp4Tabs *tabs, dim3 grid, dim3 block, hipStream_t st) {
  if (tabs)
    hipLaunchKernelGGL((link_fp4_tabs_kernel<D, NB>), grid, block, 0, st, Fp4Args{p, *tabs});
  else if (p.doc_lim)
    hipLaunchKernelGGL((link_fp4_kernel<D, true, NB>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((link_fp4_kernel<D, false, NB>), grid, block, 0, st, p);
}

}  // namespace

int fp4_rows_per_block(int max_rows) { return max_rows <= 16 ? 16 : 32; }

hipError_t launch_link_fp4(const LinkParams &p, const Fp4Tabs *tabs, hipStream_t st, const char **name) {
  *name = "link_fp4_kernel";
  const int64_t units = (int64_t)p.n_items * p.n_kv_heads;
  const dim3 grid((unsigned)unit_blocks(units, p.nrb, p.n_xcd, 0)), block(64 * kWaves);
  const bool two = fp4_rows_per_block(p.max_rows) == 32;
  if (p.d_k == 128)
    two ? launch<128, 2>(p, tabs, grid, block, st) : launch<128, 1>(p, tabs, grid, block, st);
  else
    two ? launch<64, 2>(p, tabs, grid, block, st) : launch<64, 1>(p, tabs, grid, block, st);
  return hipGetLastError();
}

}  // namespace pic
