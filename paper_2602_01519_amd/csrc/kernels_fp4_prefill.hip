// Link attention over a 4-bit chunk cache on gfx950 for calls with many rows
// per kv head, head dims 64 and 128.
//
// Workgroup: 8 waves x 32 rows = 256 rows (query token x query head) of one
// (request, kv head) over a piece of its keys, in 64-key tiles. Per tile and wave
//   S^T[64 keys][32 rows] = K . Q^T      2 x D/16 v_mfma_f32_32x32x16_bf16
//   O^T[D][32 rows]      += V^T . P^T    4 x D/32 of them
// A tile is widened once per workgroup: waves 0-3 take its keys, waves 4-7 its
// values, 1 / 8 D bytes per lane, into registers while the tile before is
// computed, then through the scaled conversion into LDS as bf16 (K rows, V
// transposed; 32 KB for D = 128, two buffers). Widening in every wave instead would read an
// eighth of the LDS bytes and convert eight times as often: 128 conversions and 64
// permutes per wave and tile beside some 130 vector instructions of the
// softmax. The own KV is bf16 and takes the same way without the conversion,
// straight from k_self / v_self.
//
// The order of the keys within a tile is free: the scores that lane (n, g) holds
// after the first product, keys 8 a + 4 g + c, are made the 8 neighbouring
// positions of its operand of the second one by where V's keys are written.
//
// Softmax: log2 domain, against the running max as it stands; a tile is redone
// against the new one when a lane's probabilities sum to more than 2^20, and the
// first tile in which a row sees a key always is. Sums are fp32 of the probabilities
// before they are rounded to bf16 for the product. (Sums that leave the fp32 range: fp4_bias.)
//
// Bound by the issue of a SIMD that its two waves share: matrix instructions are busy 48% of
// the cycles and vector ones issue in 42% (16 requests of 512 tokens over 8..20 links of 1024,
// 32/8 heads x 128: 1.72 ms, 1144 TFLOP/s; 64-wide heads, 8 requests over 16 links, 900). The next
// tile's scores formed between this one's probabilities, in a second set of registers,
// measured the same (1727 against 1711 us), although no wave waited for LDS any more;
// without barriers and widening that would take 1510 us.
#include <cfloat>

#include "fp4.hpp"

namespace pic {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8;
constexpr int kRowsPerWave = 32;
constexpr int kRows = kWaves * kRowsPerWave;
constexpr float kJumpSum = 1048576.0f;
constexpr int kQkAhead = 5;    // K-fragment read lead, in QK steps
constexpr int kPvAhead = 8;    // V-fragment read lead, in PV MFMAs

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8, u); }
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float half_swap_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_swap_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// LDS tiles in 16-byte chunks, XOR-swizzled within a row so that the fragment
// reads (16 lanes: 16 rows of K, or of V^T, at one chunk) meet no bank twice.
//   K   [key][D/8 chunks]: D = 128: c ^ (bits 2 and 3 of key & 15 swapped);
//       D = 64, two rows to 256 bytes: c ^ ((key >> 1) & 7)
//   V^T [channel][8 chunks of 8 key positions]: c ^ ((x ^ x >> 3) & 7), x = channel & 31
template <int D>
__device__ __forceinline__ int k_slot(int key, int c) {
  if constexpr (D == 128)
    return key * 16 + (c ^ ((key & 3) | ((key & 8) >> 1) | ((key & 4) << 1)));
  else
    return key * 8 + (c ^ ((key >> 1) & 7));
}
__device__ __forceinline__ int v_slot(int ch, int c) {
  const int x = ch & 31;
  return ch * 8 + (c ^ ((x ^ (x >> 3)) & 7));
}

// A copy of x that the compiler takes for another value: what is formed from it stays where
// it is used and takes no register in the loop over the tiles.
template <typename T>
__device__ __forceinline__ T fresh(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A key tile: workgroup-uniform facts.
struct TileRef {
  const char *p;     // the tile in the cache (kv head applied)
  int nvalid;        // valid keys
  int j0;            // own tiles: first own key
  int tok;           // document tiles: first row within the request's linked rows
  int own;
};

template <int D>
struct Ctx {
  ReqEntry R;
  int kvh, heads, wave, lane, n, g;
  LinkCursor<D == 64> cur;
  const char *ks, *vs;     // k_self / v_self, kv head applied, token 0 of the batch
  int64_t stride;          // ... bytes per token
  uint32_t load;           // byte offsets of this lane's share within a cache tile: codes
                           // (low half), scales
  uint32_t put;            // ... and of its first chunk within the LDS tile

  // Tile t of the request (t only grows across calls). The own link's tok0 is its
  // first row in k_self.
  __device__ __forceinline__ TileRef tile(int t) {
    while (t >= cur.end) cur.next();
    const int tt = t - cur.tile0;
    TileRef r;
    r.own = t >= R.doc_tiles;
    r.nvalid = min(kTile, cur.len - tt * kTile);
    r.j0 = tt * kTile;
    r.tok = cur.tok0 + (r.own ? 0 : tt * kTile);
    r.p = cur.base + ((int64_t)tt * heads + kvh) * Fp4Tile<D>::kBytes;
    return r;
  }
};

// This lane's share of a cache tile, as loaded: waves 0-3 the key 16 b + m (D/4
// elements from D/4 * g on), waves 4-7 the keys 16 b + 4 g ..+3 (D/16 channels from
// D/16 * m on).
template <int D>
struct Share {
  uint32_t x[D / 32];
  uint32_t scale;
};

// Keys: wave b, lane (g, m). Values: lane (m', 4 b + g), m = 4 wave + m', so that
// sixteen lanes write one whole row of V^T.
struct Place {
  bool value;
  int b, g, m;
};
template <int D>
__device__ __forceinline__ Place place(const Ctx<D> &c, int lane) {
  const int w = c.wave & 3, lo = lane & 15, hi = lane >> 4;
  const bool value = c.wave >= 4;
  return Place{value, value ? lo >> 2 : w, value ? lo & 3 : hi, value ? 4 * w + hi : lo};
}

// This lane's offsets, formed once. The chunks that it writes follow from the first:
// key chunk j of its row is the first with j exchanged into the chunk's bits, and channel
// c of its D/16 is c rows on, with c exchanged into them (both swizzles are linear).
template <int D>
__device__ __forceinline__ void set_offsets(Ctx<D> &c) {
  typedef Fp4Tile<D> T;
  const Place l = place(c, c.lane);
  const int unit = D == 128 ? (l.b * 64 + l.g * 16 + l.m) * 16
                            : ((l.b >> 1) * 64 + l.g * 16 + l.m) * 16 + (l.b & 1) * 8;
  const int key = 16 * l.b + (l.value ? 4 * l.g : l.m);
  c.load = ((l.value ? T::kV : 0) + unit) |
           (l.value ? T::v_scale(key, l.m * (D / 16) / 32) : T::k_scale(key, l.g * (D / 4) / 32)) << 16;
  c.put = l.value ? 16 * v_slot(l.m * (D / 16), 2 * l.b + (l.g & 1)) + 8 * (l.g >> 1)
                  : 16 * k_slot<D>(key, l.g * (D / 32));
}

template <int D>
__device__ __forceinline__ void fetch(const Ctx<D> &c, const TileRef &r, Share<D> &s) {
  if (r.own) {
    if (D == 128) return;       // loaded where it is written (see stage_own)
    // The same, but one word of each line here, so that it comes from the L2 then:
    // every lane a quarter of a row. (The 128-wide kernel loses 0.5% by it.)
    const Place l = place(c, fresh(c.lane));
    const int key = l.value ? 16 * l.b + 4 * l.g + (l.m & 3) : 16 * l.b + l.m;
    const int at = (l.value ? l.m >> 2 : l.g) * (D / 2);
    s.x[0] = *(const uint32_t *)((l.value ? c.vs : c.ks) +
                                 ((int64_t)r.tok + r.j0 + min(key, r.nvalid - 1)) * c.stride + at);
    return;
  }
  // (fresh: extended to 64 bits here, not kept so)
  const uint32_t at = fresh(c.load), code = at & 0xffffu, scale = at >> 16;
  if constexpr (D == 128) {
    const uint4 u = *(const uint4 *)(r.p + code);
    s.x[0] = u.x, s.x[1] = u.y, s.x[2] = u.z, s.x[3] = u.w;
  } else {
    const uint2 u = *(const uint2 *)(r.p + code);
    s.x[0] = u.x, s.x[1] = u.y;
  }
  if (c.wave >= 4)
    s.scale = *(const uint32_t *)(r.p + scale);
  else
    s.scale = *(const uint8_t *)(r.p + scale);
}

// Pairs of channels (2 kC, 2 kC + 1) of four keys into V^T as four keys of each.
template <int kC>
__device__ __forceinline__ void put_pair(uint32_t put, uint4 *vt, const uint32_t (&d)[4]) {
  char *const p = (char *)vt;
  *(uint2 *)(p + ((put ^ (32 * kC)) + 256 * kC)) =
      make_uint2(__builtin_amdgcn_perm(d[1], d[0], 0x05040100u),
                 __builtin_amdgcn_perm(d[3], d[2], 0x05040100u));
  *(uint2 *)(p + ((put ^ (32 * kC + 16)) + 256 * kC + 128)) =
      make_uint2(__builtin_amdgcn_perm(d[1], d[0], 0x07060302u),
                 __builtin_amdgcn_perm(d[3], d[2], 0x07060302u));
}

template <int D, int kC>
__device__ __forceinline__ void widen_pair(uint32_t put, const Share<D> &s, const float (&sc)[4],
                                           uint4 *vt) {
  uint32_t d[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (D == 128)
      d[i] = fp4_pair<kC>(s.x[i], sc[i]);
    else
      d[i] = (i & 1) ? fp4_pair<2 + (kC & 1)>(s.x[i >> 1], sc[i]) : fp4_pair<kC & 1>(s.x[i >> 1], sc[i]);
  }
  put_pair<kC>(put, vt, d);
}

// An own tile, from k_self / v_self straight to LDS. (Loaded a tile ahead as the
// cache's tiles are, it would hold 16 registers over the whole tile, more than
// there are; a request has few own tiles.) Keys past the last own one: the last
// key again, and zeros for values (their probability is 0, and 0 times an
// infinity would be a NaN).
template <int D>
__device__ __forceinline__ void stage_own(const Ctx<D> &c, const TileRef &r, uint4 *kt, uint4 *vt) {
  const Place l = place(c, fresh(c.lane));
  const uint32_t put = fresh(c.put);
  const char *kv = (l.value ? c.vs : c.ks) + ((int64_t)r.tok + r.j0) * c.stride;
  if (!l.value) {
    const int key = 16 * l.b + l.m;
    const char *p = kv + min(key, r.nvalid - 1) * c.stride + l.g * (D / 2);
    uint4 x[D / 32];
#pragma unroll
    for (int j = 0; j < D / 32; ++j) x[j] = *(const uint4 *)(p + 16 * j);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) *(uint4 *)((char *)kt + (put ^ (16 * j))) = x[j];
    return;
  }
  uint32_t x[D / 32][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = 16 * l.b + 4 * l.g + i;
    const char *p = kv + min(key, r.nvalid - 1) * c.stride + l.m * (D / 8);
    const uint32_t keep = key < r.nvalid ? ~0u : 0u;
#pragma unroll
    for (int j = 0; j < D / 32; j += 2) {
      const uint2 u = *(const uint2 *)(p + 4 * j);
      x[j][i] = u.x & keep;
      x[j + 1][i] = u.y & keep;
    }
  }
  put_pair<0>(put, vt, x[0]);
  put_pair<1>(put, vt, x[1]);
  if constexpr (D == 128) {
    put_pair<2>(put, vt, x[2]);
    put_pair<3>(put, vt, x[3]);
  }
}

template <int D>
__device__ __forceinline__ void widen(const Ctx<D> &c, const TileRef &r, const Share<D> &s, uint4 *kt,
                                      uint4 *vt) {
  if (r.own) {
    if (D == 64) asm volatile("" ::"v"(s.x[0]));
    stage_own(c, r, kt, vt);
    return;
  }
  const uint32_t put = D == 64 ? fresh(c.put) : c.put;   // (fragment addresses: see compute_tile)
  if (c.wave < 4) {
    const float sc = fp4_scale(s.scale);
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
      *(uint4 *)((char *)kt + (put ^ (16 * j))) = fp4_decode8(s.x[j], sc);
    return;
  }
  float sc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sc[i] = fp4_scale((s.scale >> (8 * i)) & 255u);
  widen_pair<D, 0>(put, s, sc, vt);
  widen_pair<D, 1>(put, s, sc, vt);
  if constexpr (D == 128) {
    widen_pair<D, 2>(put, s, sc, vt);
    widen_pair<D, 3>(put, s, sc, vt);
  }
}

template <int D>
struct Acc {
  f32x16 o[D / 32];
  float m, l;      // running max in use (log2 domain); this lane half's part of the sum
};

// Per-row limit on the visible linked rows, and its minimum over the wave.
struct DocLim {
  int dl, wmin;
};

// own_last(): last own key that this lane's row sees (formed where a tile needs it). jump:
// the lane's sum of probabilities above which a tile is redone; bias: added to its maximum.
template <int D, bool kLim, class OwnLast>
__device__ __forceinline__ void compute_tile(const Ctx<D> &c, const uint4 *kt, const uint4 *vt,
                                             const bf16x8 (&qf)[D / 16], Acc<D> &a, const TileRef &r,
                                             OwnLast own_last, const DocLim &dlm, float sc,
                                             float jump, float bias) {
  f32x16 s0, s1;
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    s0[x] = 0.f;
    s1[x] = 0.f;
  }
  // Fragment addresses: chunk 2 st + g of a row is the row's chunk g with the bits
  // of st exchanged. (D = 64 forms them for every tile: kept, they would take
  // the registers that let two workgroups share a CU.)
  uint32_t kbase = 16 * k_slot<D>(c.n, c.g), vbase = 16 * v_slot(c.n, c.g);
  if (D == 64) kbase = fresh(kbase), vbase = fresh(vbase);
  auto k_frag = [&](int half, int st) {
    return as_bf16x8(*(const uint4 *)((const char *)kt + ((kbase ^ (st << 5)) + half * 64 * D)));
  };
  auto v_frag = [&](int d, int ks) {
    return as_bf16x8(*(const uint4 *)((const char *)vt + ((vbase ^ (ks << 5)) + d * 4096)));
  };
  constexpr int kSteps = D / 16, kAhead = D == 64 ? 4 : kQkAhead;
  bf16x8 ka[kSteps], kb[kSteps];
#pragma unroll
  for (int st = 0; st < kAhead; ++st) {
    ka[st] = k_frag(0, st);
    kb[st] = k_frag(1, st);
  }
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    if (st + kAhead < kSteps) {
      ka[st + kAhead] = k_frag(0, st + kAhead);
      kb[st + kAhead] = k_frag(1, st + kAhead);
    }
    s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[st], qf[st], s0, 0, 0, 0);
    s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[st], qf[st], s1, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  // s0[x] / s1[x]: key 8 (x >> 2) + 4 g + (x & 3) (+ 32)
  if (r.own || r.nvalid < kTile || (kLim && r.tok + kTile > dlm.wmin)) {
    int kl = kLim ? min(dlm.dl - r.tok, r.nvalid) - 1 : r.nvalid - 1;
    if (r.own) kl = min(own_last() - r.j0, r.nvalid - 1);
    kl -= 4 * (fresh(c.lane) >> 5);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      // (opaque: the compiler otherwise chains the comparisons through some
      // sixty scalar registers, and spills those of the loop)
      int k = kl;
      asm volatile("" : "+v"(k));
      const int key = 8 * (x >> 2) + (x & 3);
      if (key > k) s0[x] = -INFINITY;
      if (key + 32 > k) s1[x] = -INFINITY;
    }
  }
  bf16x8 pf[4];
  auto probs = [&]() {
    const float neg_m = a.m == -INFINITY ? 0.f : -a.m;
    float t0 = 0.f, t1 = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s0[x], sc, neg_m));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1[x], sc, neg_m));
      t0 += p0;
      t1 += p1;
      pf[x >> 3][x & 7] = (__bf16)p0;
      pf[2 + (x >> 3)][x & 7] = (__bf16)p1;
    }
    return t0 + t1;
  };
  auto tile_max = [&]() {
    float t = -INFINITY;
#pragma unroll
    for (int x = 0; x < 16; ++x) t = fmaxf(fmaxf(t, s0[x]), s1[x]);
    return t;
  };
  float ts = probs();
  bool redo = !(ts <= jump);
  // A row that has seen no key yet and sees one here (its probabilities against a
  // maximum of 0 may all be 0).
  if (__builtin_expect(__any(a.m == -INFINITY), 0)) redo |= a.m == -INFINITY && tile_max() > -INFINITY;
  if (__builtin_expect(__any(redo), 0)) {
    const float tmax = half_swap_max(tile_max());
    const float mnew = fmaxf(a.m, __builtin_fmaf(tmax, sc, bias));
    const float alpha = mnew == a.m ? 1.f : __builtin_amdgcn_exp2f(a.m - mnew);
    a.m = mnew;
    a.l *= alpha;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int x = 0; x < 16; ++x) a.o[d][x] *= alpha;
    ts = probs();
  }
  a.l += ts;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      a.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(d, ks), pf[ks], a.o[d], 0, 0, 0);
    }
  // V reads run kPvAhead MFMAs ahead
  constexpr int kPv = D / 8, kVAhead = kPvAhead;
  __builtin_amdgcn_sched_group_barrier(0x100, kVAhead, 0);
#pragma unroll
  for (int i = 0; i < kPv; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + kVAhead < kPv) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
}

// big: the second pass (see fp4_bias). Returns whether the workgroup's sums left the fp32 range
// in the first one (and nothing was written).
template <int D, bool kLim, bool kArg>
__device__ __forceinline__ bool link_body(int wave, bool big) {
  const Fp4Start<kArg> start(wave);
  const LinkParams &p = start.p;
  // one array, so that a lane's address serves both buffers
  __shared__ uint4 lds[4][kTile * D / 8];
  __shared__ int over[kWaves];     // per wave: its sums left the fp32 range
  uint4 *const sk0 = lds[0], *const sk1 = lds[1], *const sv0 = lds[2], *const sv1 = lds[3];
  Ctx<D> c;
  c.lane = start.lane;
  c.wave = start.wave;
  c.n = c.lane & 31;
  c.g = c.lane >> 5;
  const int units = p.n_items * p.n_kv_heads;
  const UnitBlock ub = unit_of_block(start.block, p.nrb, p.n_xcd, p.spread, units);
  const int rb = ub.rb;
  if (ub.u >= units) return false;
  const WorkItem it = load_item(start.items, ub.u / p.n_kv_heads);
  c.heads = p.n_kv_heads;
  c.kvh = ub.u % p.n_kv_heads;
  c.R = item_request(it);
  const ReqEntry &R = c.R;
  const int group = p.group;
  const int nrows = R.lq * group;
  const int row0 = rb * kRows;
  if (row0 >= nrows) return false;
  const int vis = visible_tiles(R, min(nrows - 1, row0 + kRows - 1) / group);
  const int t_begin = it.t_begin;
  int t_end = min(it.t_end, vis);
  if (kLim && R.ls == 0 && t_begin < t_end)
    t_end = limit_end(p, it, R.q0 + row0 / group, R.q0 + min(nrows - 1, row0 + kRows - 1) / group,
                      c.lane, t_end);

  // this lane's row; a wave without rows only widens its share of every tile
  const bool active = row0 + c.wave * kRowsPerWave < nrows;
  const int row = row0 + c.wave * kRowsPerWave + c.n;
  auto own_last = [&]() {
    const int r = row0 + c.wave * kRowsPerWave + (fresh(c.lane) & 31);
    return r < nrows ? r / group + R.ls - R.lq : -1;
  };
  // row of q and out (formed again after the loop over the tiles, which it would
  // cost registers)
  auto out_row = [&](int lane) {
    const int r = row0 + c.wave * kRowsPerWave + (lane & 31);
    const int i = r < nrows ? r / group : 0;
    return (int64_t)(R.q0 + i) * p.n_q_heads + c.kvh * group + (r < nrows ? r % group : 0);
  };
  DocLim dlm{kNoLimit, kNoLimit};
  if (kLim) {
    if (row < nrows) dlm.dl = p.doc_lim[R.q0 + row / group];
    int w = dlm.dl;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) w = min(w, __shfl_xor(w, o));
    dlm.wmin = uni(w);
  }
  c.cur.start(start.links, it);
  set_offsets(c);
  c.stride = (int64_t)p.n_kv_heads * D * 2;
  c.ks = (const char *)p.k_self + c.kvh * D * 2;
  c.vs = (const char *)p.v_self + c.kvh * D * 2;

  TileRef ref0{}, ref1{};
  Share<D> sh{};
  if (t_begin < t_end) {
    ref0 = c.tile(t_begin);
    fetch(c, ref0, sh);
  }
  bf16x8 qf[D / 16];
  {
    const uint4 *qrow = (const uint4 *)((const uint16_t *)p.q + out_row(c.lane) * D);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row < nrows) v = qrow[s * 2 + c.g];
      qf[s] = as_bf16x8(v);
    }
  }
  Acc<D> a;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int x = 0; x < 16; ++x) a.o[d][x] = 0.f;
  a.m = -INFINITY;
  a.l = 0.f;
  const float sc = p.scale_log2;
  const float bias = big ? fp4_bias(max(1, t_end - t_begin)) : 0.f, jump = big ? 0.f : kJumpSum;

  if (t_begin < t_end) {
    widen(c, ref0, sh, sk0, sv0);
    __syncthreads();
  }
  // The queries have landed: without this use the loop's first products wait for
  // every load in flight, the next tile's among them.
#pragma unroll
  for (int s = 0; s < D / 16; ++s) asm volatile("" : "+v"(qf[s]));
  // Tile t is computed from one buffer pair while tile t + 1 is loaded into
  // registers and then widened into the other (past the last tile: the last one
  // again, into the buffers nobody reads); unrolled by two so that every access
  // names its buffers.
  for (int t = t_begin; t < t_end; t += 2) {
    ref1 = t + 1 < t_end ? c.tile(t + 1) : ref0;
    fetch(c, ref1, sh);
    if (active) compute_tile<D, kLim>(c, sk0, sv0, qf, a, ref0, own_last, dlm, sc, jump, bias);
    widen(c, ref1, sh, sk1, sv1);
    __syncthreads();
    if (t + 1 >= t_end) break;
    ref0 = t + 2 < t_end ? c.tile(t + 2) : ref1;
    fetch(c, ref0, sh);
    if (active) compute_tile<D, kLim>(c, sk1, sv1, qf, a, ref1, own_last, dlm, sc, jump, bias);
    widen(c, ref0, sh, sk0, sv0);
    __syncthreads();
  }

  if (!big) {
    float most = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int x = 0; x < 16; ++x) most = __builtin_elementwise_maximum(most, fabsf(a.o[d][x]));
    const bool mine = __any(!(most <= FLT_MAX));
    if (c.lane == 0) over[c.wave] = mine;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) any |= over[w];
    if (__builtin_expect(any, 0)) return true;
  }

  // ---- epilogue: O^T[dv][row], dv = 32 d + 8 (x >> 2) + 4 g + (x & 3)
  const int lane = fresh(c.lane);
  const bool rvalid = row0 + c.wave * kRowsPerWave + (lane & 31) < nrows;
  const int64_t orow = out_row(lane);
  const float ltot = half_swap_sum(a.l);
  const int nvalid = min(kRowsPerWave, nrows - (row0 + c.wave * kRowsPerWave));
  if (nvalid <= 0) return false;
  const float inv = ltot > 0.f ? 1.f / ltot : 0.f;
  const int64_t prow = it.part + (orow - (int64_t)R.q0 * p.n_q_heads);
  if constexpr (D == 128) {
    typedef __attribute__((address_space(3))) void *lds_ptr;
    const int bi = c.wave & 3;
    const lds_ptr buf = bi == 0 ? (lds_ptr)sk0 : bi == 1 ? (lds_ptr)sk1 : bi == 2 ? (lds_ptr)sv0 : (lds_ptr)sv1;
    const lds_units sb =
        (lds_units)(uintptr_t)((uint32_t)(uintptr_t)buf + (c.wave >> 2) * kStoreBytes);
    if (it.part < 0)
      store_block_bf16(a.o[0], a.o[1], a.o[2], a.o[3], inv, sb, c.lane, nvalid, (int)orow,
                       (uint16_t *)p.out, D);
    else if (!p.skip_empty || __any(!(ltot == 0.f)))
      store_block_f32(a.o[0], a.o[1], a.o[2], a.o[3], sb, c.lane, nvalid, (int)prow, p.part_o, D);
  } else if (rvalid) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int dv = 32 * d + 8 * j + 4 * c.g;
        if (it.part < 0) {
          bf16x4v v;
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] = (__bf16)(a.o[d][4 * j + x] * inv);
          *(uint2 *)((uint16_t *)p.out + orow * D + dv) = __builtin_bit_cast(uint2, v);
        } else {
          *(float4 *)(p.part_o + prow * D + dv) =
              make_float4(a.o[d][4 * j], a.o[d][4 * j + 1], a.o[d][4 * j + 2], a.o[d][4 * j + 3]);
        }
      }
  }
  if (!rvalid || c.g != 0) return false;
  if (it.part < 0) {
    if (p.lse) p.lse[orow] = ltot == 0.f ? -INFINITY : log_sum(a.m, ltot);
  } else {
    p.part_m[prow] = partial_max(a.m, ltot);
    p.part_l[prow] = ltot;
  }
  return false;
}

template <int D, bool kLim, bool kArg>
__device__ __forceinline__ void link_piece() {
  const int wave = uni(threadIdx.x >> 6);
  for (bool big = false; link_body<D, kLim, kArg>(wave, big); big = true) {
  }
}

template <int D, bool kLim>
__global__ __launch_bounds__(kWaves * 64, D == 64 ? 4 : 2) void link_fp4_prefill_kernel(LinkParams) {
  link_piece<D, kLim, false>();
}
// The tables are read where they are, in the kernel arguments.
template <int D>
__global__ __launch_bounds__(kWaves * 64, D == 64 ? 4 : 2) void link_fp4_prefill_tabs_kernel(Fp4Args) {
  link_piece<D, false, true>();
}

template <int D>
hipError_t launch(const LinkParams &p, const Fp4Tabs *tabs, hipStream_t st) {
  const int64_t units = (int64_t)p.n_items * p.n_kv_heads;
  const dim3 grid((unsigned)unit_blocks(units, p.nrb, p.n_xcd, p.spread)), block(kWaves * 64);
  if (tabs)
    hipLaunchKernelGGL(link_fp4_prefill_tabs_kernel<D>, grid, block, 0, st, Fp4Args{p, *tabs});
  else if (p.doc_lim)
    hipLaunchKernelGGL((link_fp4_prefill_kernel<D, true>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((link_fp4_prefill_kernel<D, false>), grid, block, 0, st, p);
  return hipGetLastError();
}

}  // namespace

int fp4_prefill_rows_per_block() { return kRows; }
// resident workgroups per CU (two or four waves per SIMD)
int fp4_prefill_blocks_per_cu(int d) { return d == 64 ? 2 : 1; }

hipError_t launch_link_fp4_prefill(const LinkParams &p, const Fp4Tabs *tabs, hipStream_t st,
                                   const char **name) {
  *name = "link_fp4_prefill_kernel";
  return p.d_k == 128 ? launch<128>(p, tabs, st) : launch<64>(p, tabs, st);
}

}  // namespace pic
