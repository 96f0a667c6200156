// bf16 GQA link attention of requests that share links, head dim 128 or 64, on the matrix cores:
// row blocks of pieces of keys, to partials (merge_kernel joins them).
//
// Block: 256 or 128 rows (query token x head of the group) of one (item, kv head), an item a piece of
// the keys of a group of requests, of 64-wide heads also of one request with its own KV. 256: 8
// waves of 32 rows, each over whole 64-key tiles; 128: 4 groups of 32 rows x 2 halves of each tile,
// whose (m, l, O) merge through LDS at the end.
//   S^T[64 (32) keys][32 rows] = K . Q^T    D / 8 (D / 16) x v_mfma_f32_32x32x16_bf16
//   O^T[D][32 rows]           += V^T . P^T  the same
// The tiles' LDS layout, the key order of the scores and the softmax are link_mfma_d128_kernel's:
// probabilities against the running max as it stands, a tile done again against its own max where
// a sum passes 2^64 or the row has no max yet. The row sums are of the fp32 probabilities.
// 128 wide, a tile takes a CU 2.1 us at 256 rows (1000 TFLOP/s on all of them, the rate of
// link_mfma_d128_kernel) and 1.05 at 128, which groups of no more rows take. Larger groups in blocks
// of 128 would be cut into half as many pieces, with half the partials, but read each key once
// more: 64 requests x 32/8 heads over 16 links of 1024 50.8 us, in blocks of 256 45.9. 64-wide heads
// have half the products beside the same exponentials: 1.2 us a tile of 256 rows (895 TFLOP/s).
//
// Tiles are copied global -> LDS three ahead of their use (four buffers): keys that come from HBM
// arrive 2 us after their copies are issued, four tiles' products.
//
// 128-wide heads, single tokens: the requests' own links and KV have a few rows per key and are
// bound by HBM where the groups' blocks are bound by the matrix cores. Both go in one launch: the
// planner divides the CUs, some workgroups' waves take the requests' pieces one after another
// (decode_d128.hpp; own rows are read in place and turn through LDS), the others a block each.
#include <cfloat>

#include "decode_d128.hpp"

namespace pic {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void *lds_ptr;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kRowsPerWave = 32;
template <bool kWide>
constexpr int kRows = kWide ? 256 : 128;        // of a block
constexpr int kBuffers = 4;                     // tiles in LDS
template <int D>
constexpr int kUnits = kTile * D / 8;           // 16-byte units of a K (or V) tile
template <int D>
constexpr int kSets = D / 64;                   // copies a lane of each
constexpr float kJumpSum = 18446744073709551616.0f;   // 2^64
static_assert(kWaves * decode_d128::kOwnScratch <= kBuffers * 2 * kUnits<128> * 16, "LDS");

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8, u); }

// LDS tiles in 16-byte units, swizzled within each row (see link_mfma_d128_kernel): K [key][D / 8
// units of 8 dims], V^T [dv][8 units of 8 keys]. Rows of 8 units lie two to a 256-byte bank row: the
// 16 rows that a group of lanes reads, {0-3, 8-11, 4-7, 12-15}, take every unit of both.
__device__ __forceinline__ int hk(int key) { return (key & 3) | ((key & 8) >> 1) | ((key & 4) << 1); }
__device__ __forceinline__ int hv(int x) { return (x ^ (x >> 3)) & 7; }
template <int D>
__device__ __forceinline__ int k_unit(int key, int c) {      // c ^ the row's swizzle
  return D == 128 ? c ^ hk(key & 15) : c ^ hv(key & 31);
}
template <int D>
__device__ __forceinline__ int k_slot(int key, int c) { return key * (D / 8) + k_unit<D>(key, c); }
__device__ __forceinline__ int v_slot(int dv, int c) { return dv * 8 + (c ^ hv(dv & 31)); }
// Key row that feeds M index m: a lane's scores are then 8 consecutive keys, twice.
__device__ __forceinline__ int key_of_m(int m) {
  const int a = m >> 3, g = (m >> 2) & 1, c = m & 3;
  return (a >> 1) * 16 + g * 8 + (a & 1) * 4 + c;
}
__device__ __forceinline__ float half_max(float x) {     // over lanes i and i ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

struct TileRef {
  const char *k, *v;
  int nvalid;
  int own;                      // 0, or 1 + the first key's index among the own ones
};
struct Cursor {
  const_links links;            // from the item's first link on
  int li, kvh, doc_tiles;
  const char *k, *v;
  int len, lp, tile0, end;
};
__device__ __forceinline__ void cursor_set(Cursor &c, const void *k, const void *v, int len, int lp, int tile0) {
  c.k = (const char *)k;
  c.v = (const char *)v;
  c.len = len;
  c.lp = lp;
  c.tile0 = tile0;
  c.end = tile0 + (len + kTile - 1) / kTile;
}
template <int D>
__device__ __forceinline__ TileRef tile_ref(Cursor &c, int t) {   // (t only grows)
  while (t >= c.end) {
    ++c.li;
    cursor_set(c, c.links[c.li].k, c.links[c.li].v, c.links[c.li].len, c.links[c.li].lp, c.links[c.li].tile0);
  }
  const int tt = t - c.tile0;
  return TileRef{c.k + ((int64_t)c.kvh * c.lp + tt * kTile) * D * 2,
                 c.v + ((int64_t)c.kvh * D * c.lp + tt * kTile * D) * 2, min(kTile, c.len - tt * kTile),
                 t >= c.doc_tiles ? 1 + tt * kTile : 0};
}

template <int kAux>
__device__ __forceinline__ void copy16(const void *base, uint32_t off, uint4 *dst) {
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), (short)0, -1, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)dst, 16, off, 0, 0, kAux);
}

template <int D>
struct Lane {
  int lane, wave, n, g;         // n: row of the wave's 32, g: lane / 32
  int half;                     // (blocks of 128 rows) the wave's half of a tile's keys
  uint32_t koff[kSets<D>], voff[kSets<D>];      // byte offsets of the lane's K and V units within a tile
};

// Copy i of a tile into a buffer (its K units, then its V units).
template <int D, int kAux>
__device__ __forceinline__ void tile_copy(const Lane<D> &c, int i, const TileRef &r, uint4 *to) {
  constexpr int n = kSets<D>;
  if (i < n)
    copy16<kAux>(r.k, c.koff[i], to + (i * kWaves + c.wave) * 64);
  else
    copy16<kAux>(r.v, c.voff[i - n], to + kUnits<D> + ((i - n) * kWaves + c.wave) * 64);
}

template <int D>
struct State {
  f32x16 o[D / 32];
  float m, l;
};

// When a tile is done again against its own max, and what that max is raised by (64 wide, where the
// sums of a block left the fp32 range: every tile, and the logarithm of the block's keys).
struct Steps {
  float jump, raise;
};

// One tile, the copies of a later one spread over its score products. The wave takes kN halves of
// the tile's keys, from c.half on. lim: the last own key that this lane's row sees.
template <int D, int kN, int kAux>
__device__ __forceinline__ void compute_tile(const Lane<D> &c, const uint4 *kt, const bf16x8 (&qf)[D / 16], State<D> &a,
                                             const TileRef &r, int lim, float sc, Steps steps, const TileRef &next,
                                             uint4 *to) {
  const uint4 *vt = kt + kUnits<D>;
  constexpr int kSteps = D / 16, kAhead = D == 64 ? 4 : 5;   // K reads run ahead of their products
  const int row = 32 * c.half + key_of_m(c.n);
  f32x16 s[kN];
#pragma unroll
  for (int h = 0; h < kN; ++h)
#pragma unroll
    for (int x = 0; x < 16; ++x) s[h][x] = 0.f;
  bf16x8 kf[kN][kSteps];
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
#pragma unroll
    for (int h = 0; h < kN; ++h) kf[h][i] = as_bf16x8(kt[k_slot<D>(32 * h + row, i * 2 + c.g)]);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (i + kAhead < kSteps) {
#pragma unroll
      for (int h = 0; h < kN; ++h)
        kf[h][i + kAhead] = as_bf16x8(kt[k_slot<D>(32 * h + row, (i + kAhead) * 2 + c.g)]);
    }
    if (i % 2 == 0) tile_copy<D, kAux>(c, i / 2, next, to);
#pragma unroll
    for (int h = 0; h < kN; ++h) s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[h][i], qf[i], s[h], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  // s[h][x]: key 32 (half + h) + (x >> 3) * 16 + g * 8 + (x & 7)
  constexpr bool kOwn = D == 64;                // (128-wide items are of shared rows alone)
  bool seen = true;
  if (__builtin_expect(r.nvalid < kTile || (kOwn && r.own), 0)) {
    asm volatile("");             // (a branch: as selects, the masks of whole tiles cost 45 instructions)
    const int last = kOwn && r.own ? min(lim + 1 - r.own, r.nvalid - 1) : r.nvalid - 1;
    const int kl = last - 32 * c.half - 8 * c.g;
#pragma unroll
    for (int h = 0; h < kN; ++h)
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (32 * h + (x >> 3) * 16 + (x & 7) > kl) s[h][x] = -INFINITY;
    seen = kl >= 0;
  }
  bf16x8 pf[2 * kN];                            // rounded to bf16, 2^-8 of each; the sums are not
  auto probs = [&]() {
    const float neg = a.m == -INFINITY ? 0.f : -a.m;
    float t[2] = {0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int h = 0; h < kN; ++h) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][x], sc, neg));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][8 + x], sc, neg));
        pf[2 * h][x] = (__bf16)p0;
        pf[2 * h + 1][x] = (__bf16)p1;
        t[0] += p0;
        t[1] += p1;
      }
    return t[0] + t[1];
  };
  float t = probs();
  if (__builtin_expect(__any(!(t <= (D == 64 ? steps.jump : kJumpSum)) || (a.m == -INFINITY && seen)), 0)) {
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < kN; ++h)
#pragma unroll
      for (int x = 0; x < 16; x += 2) top = fmaxf(fmaxf(top, s[h][x]), s[h][x + 1]);
    top = half_max(top);
    const float mnew = fmaxf(a.m, D == 64 ? top * sc + steps.raise : top * sc);
    const float f = mnew == a.m ? 1.f : __builtin_amdgcn_exp2f(a.m - mnew);
    a.m = mnew;
    a.l *= f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int x = 0; x < 16; ++x) a.o[d][x] *= f;
    t = probs();
  }
  a.l += t;
#pragma unroll
  for (int k = 0; k < 2 * kN; ++k)
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      const bf16x8 vf = as_bf16x8(vt[v_slot(d * 32 + c.n, (2 * c.half + k) * 2 + c.g)]);
      a.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[k], a.o[d], 0, 0, 0);
    }
  constexpr int kPv = kN * D / 16, kLead = kPv / 2;   // V reads run ahead of their products
  __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
  for (int i = 0; i < kPv; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + kLead < kPv) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
}

// After a tile: the next one's copies have landed (those of the two behind it may be in flight),
// the LDS reads are done, and no access moves across.
template <int D>
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * kSets<D>) : "memory");
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int D, bool kWide, int kAux>
__device__ __forceinline__ void block_partial(const LinkParams &p, const WorkItem &it, int rb, int kvh, uint4 *lds) {
  Lane<D> c;
  c.lane = threadIdx.x & 63;
  c.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  c.n = c.lane & 31;
  c.g = c.lane >> 5;
  c.half = kWide ? 0 : c.wave & 1;
  const int rg = kWide ? c.wave : c.wave >> 1;  // (the waves of few rows: one on each SIMD)
  const int group = p.group, nrows = it.lq * group, row0 = rb * kRows<kWide>;
  const bool active = row0 + rg * kRowsPerWave < nrows;
  const int row = row0 + rg * kRowsPerWave + c.n;
  const bool rvalid = row < nrows;
  const int qi = rvalid ? row / group : 0, qh = kvh * group + (rvalid ? row % group : 0);
  const int64_t orow = (int64_t)(it.q0 + qi) * p.n_q_heads + qh;
#pragma unroll
  for (int u = 0; u < kSets<D>; ++u) {          // (load-to-LDS: lane i lands at unit base + i)
    const int s = (u * kWaves + c.wave) * 64 + c.lane;
    const int key = s / (D / 8), kc = k_unit<D>(key, s % (D / 8));
    c.koff[u] = (uint32_t)((key * D + kc * 8) * 2);
    const int dv = s >> 3, cc = (s & 7) ^ hv(dv & 31);
    c.voff[u] = (uint32_t)((cc >> 2) * D * kPanel * 2 + dv * kPanel * 2 + (cc & 3) * 16);
  }
  Cursor cur;
  cur.links = (const_links)p.links + it.link;
  cur.li = 0;
  cur.kvh = kvh;
  cur.doc_tiles = it.doc_tiles;
  cursor_set(cur, it.k, it.v, it.len, it.lp, it.tile0);
  const int lim = rvalid ? qi + it.ls - it.lq : -1;
  // own tiles past the causal limit of the block's last row hold no key that it sees
  const int t0 = it.t_begin;
  const int t1 = D == 128 ? it.t_end
                          : min(it.t_end, visible_tiles(item_request(it), (min(nrows, row0 + kRows<kWide>) - 1) / group));
  // (past the last tile the copies repeat it into buffers nobody reads again, which keeps the
  // counts of the waits)
  Steps steps{kJumpSum, 0.f};
  TileRef r0{}, r1{}, r2{}, r3{};
  auto tile = [&](int t) { return tile_ref<D>(cur, min(t, t1 - 1)); };
  auto issue = [&](const TileRef &r, int i) {
#pragma unroll
    for (int k = 0; k < 2 * kSets<D>; ++k) tile_copy<D, kAux>(c, k, r, lds + 2 * kUnits<D> * i);
  };
  if (t0 < t1) {
    r0 = tile(t0);
    issue(r0, 0);
  }
  bf16x8 qf[D / 16];
  {
    const uint4 *q = (const uint4 *)((const uint16_t *)p.q + orow * D);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (rvalid) v = q[s * 2 + c.g];
      qf[s] = as_bf16x8(v);
    }
  }
  State<D> a;
  const auto clear = [&]() {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int x = 0; x < 16; ++x) a.o[d][x] = 0.f;
    a.m = -INFINITY;
    a.l = 0.f;
  };
  clear();
  const auto restart = [&]() {
    clear();
    cur.li = 0;
    cursor_set(cur, it.k, it.v, it.len, it.lp, it.tile0);
    r0 = tile(t0);
    issue(r0, 0);
  };
  const float sc = p.scale_log2;
  const auto walk = [&]() {                     // the first tile's copies are on their way
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    // (behind the first tile's arrival, which they would delay)
    r1 = tile(t0 + 1);
    issue(r1, 1);
    r2 = tile(t0 + 2);
    issue(r2, 2);
    // Tile t from buffer i, the copies of tile t + 3 into the one that tile t - 1 left.
    auto step = [&](const TileRef &r, int i, const TileRef &next) {
      if (active)
        compute_tile<D, kWide ? 2 : 1, kAux>(c, lds + 2 * kUnits<D> * i, qf, a, r, lim, sc, steps, next,
                                             lds + 2 * kUnits<D> * ((i + 3) & 3));
      else
        issue(next, (i + 3) & 3);
      tile_barrier<D>();
    };
    for (int t = t0; t < t1; t += 4) {
      r3 = tile(t + 3);
      step(r0, 0, r3);
      if (t + 1 >= t1) break;
      r0 = tile(t + 4);
      step(r1, 1, r0);
      if (t + 2 >= t1) break;
      r1 = tile(t + 5);
      step(r2, 2, r1);
      if (t + 3 >= t1) break;
      r2 = tile(t + 6);
      step(r3, 3, r2);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                            // every copy has landed, every tile is done with
  };
  if (t0 < t1) {
#pragma unroll 1
    for (;;) {
      walk();
      if constexpr (D == 128) break;            // (values up to 2^61 / tiles: see pic.h)
      // Probabilities against a max that lags reach 2^64: the sums of large values may leave the
      // fp32 range, of 128 rows also only where the two halves of the keys are joined. Then once
      // more, against a max that keeps them below the largest value.
      constexpr float kMost = kWide ? FLT_MAX : FLT_MAX / 2;
      float most = 0.f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) most = __builtin_elementwise_maximum(most, fabsf(a.o[d][x]));   // (NaN if one is)
      if (steps.raise > 0.f || !__syncthreads_or(!(most <= kMost))) break;
      steps = Steps{0.f, ceilf(log2f((float)(t1 - t0))) + 6.f};
      restart();
    }
  }

  const int nvalid = min(kRowsPerWave, nrows - (row0 + rg * kRowsPerWave));
  const int64_t prow = it.part + (orow - (int64_t)it.q0 * p.n_q_heads);
  // 64 dims of the wave's rows (O^T[dv][row], dv = d * 32 + (x >> 2) * 8 + g * 4 + (x & 3)) leave
  // through 8 KB of LDS as whole 256-byte pieces
  auto store = [&](const f32x16 &o0, const f32x16 &o1, float *lds8k, int dim0) {
    const lds_units units = (lds_units)(uintptr_t)(uint32_t)(uintptr_t)(lds_ptr)lds8k;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const f32x16 &o = d ? o1 : o0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        units[c.n * 16 + ((8 * d + 2 * j + c.g) ^ (c.n & 15))] = __builtin_bit_cast(
            u32x4v, (f32x4v){o[j * 4], o[j * 4 + 1], o[j * 4 + 2], o[j * 4 + 3]});
    }
    store_block_units(units, c.lane, nvalid, (int)prow, (char *)(p.part_o + dim0), D * 4);
  };
  float *xo = (float *)lds, *mine = xo + c.wave * 2048;
  if constexpr (kWide) {
    if (!active) return;
    const float sum = half_sum(a.l);
    if constexpr (D == 128)
      store_block_f32(a.o[0], a.o[1], a.o[2], a.o[3], (lds_units)(uintptr_t)(uint32_t)(uintptr_t)(lds_ptr)mine, c.lane,
                      nvalid, (int)prow, p.part_o, D);
    else
      store(a.o[0], a.o[1], mine, 0);
    if (rvalid && c.g == 0) {
      p.part_m[prow] = partial_max(a.m, sum);
      p.part_l[prow] = sum;
    }
    return;
  }

  // The halves of a row group merge: each wave hands over the two 32-dim blocks that the other
  // writes out (64 wide: the second half all it has; 8 KB a wave, same lanes on both sides), and
  // its max and sum behind them.
  float *xm = xo + kWaves * 2048;
  const int other = c.wave ^ 1;
  const float *theirs = xo + other * 2048;
  constexpr bool kBoth = D == 128;              // both halves write out
  const int give = kBoth && !c.half ? 2 : 0, keep = kBoth && c.half ? 2 : 0;
  const bool gives = active && (kBoth || c.half), keeps = active && (kBoth || !c.half);
  if (gives) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const f32x16 &o = kBoth && give ? a.o[(D / 32 - 2) + d] : a.o[d];
        *(float4 *)(mine + ((d * 4 + x / 4) * 64 + c.lane) * 4) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
      }
    xm[c.wave * 128 + c.lane] = a.m;
    xm[c.wave * 128 + 64 + c.lane] = a.l;
  }
  __syncthreads();
  f32x16 s0, s1;                                // the wave's 64 dims, merged
  float m = -INFINITY, l = 0.f;
  if (keeps) {
    const float m1 = xm[other * 128 + c.lane], l1 = xm[other * 128 + 64 + c.lane];
    m = fmaxf(a.m, m1);
    const float f0 = a.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.m - m);
    const float f1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - m);
    // (a NaN score leaves a NaN sum beside a max that may be -inf: it stays)
    l = (a.m == -INFINITY ? a.l : a.l * f0) + (m1 == -INFINITY ? l1 : l1 * f1);
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const f32x16 &o = kBoth && keep ? a.o[(D / 32 - 2) + d] : a.o[d];
      f32x16 &to = d ? s1 : s0;
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const float4 v = *(const float4 *)(theirs + ((d * 4 + x / 4) * 64 + c.lane) * 4);
        to[x] = o[x] * f0 + v.x * f1;
        to[x + 1] = o[x + 1] * f0 + v.y * f1;
        to[x + 2] = o[x + 2] * f0 + v.z * f1;
        to[x + 3] = o[x + 3] * f0 + v.w * f1;
      }
    }
  }
  __syncthreads();                              // the exchange is over: 8 KB of it for each wave
  if (keeps) {
    store(s0, s1, mine, 32 * keep);
    const float sum = half_sum(l);
    if (rvalid && c.g == 0 && c.half == 0) {
      p.part_m[prow] = partial_max(m, sum);
      p.part_l[prow] = sum;
    }
  }
}

// The first unit_wgs workgroups take the wave units, the others a block each.
template <int D, bool kWide, int kAux>
__global__ __launch_bounds__(kThreads, 1) void link_shared_kernel(SharedParams p) {
  __shared__ uint4 lds[kBuffers * 2 * kUnits<D> + (D == 64 ? 512 : 0)];   // (64 wide: the exchange is larger)
  if (D == 128 && (int)blockIdx.x < p.unit_wgs) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int u = blockIdx.x + p.unit_wgs * wave; u < p.n_units; u += p.unit_wgs * kWaves)
      decode_d128::wave_unit<true, true>(p.own, u, lane, (char *)lds + wave * decode_d128::kOwnScratch);
    return;
  }
  const int x = blockIdx.x - p.unit_wgs, b = x / p.pre.n_kv_heads;
  typedef __attribute__((address_space(4))) const SharedBlock *const_blocks;
  const int rb = ((const_blocks)p.blocks + b)->rb;
  block_partial<D, kWide, kAux>(p.pre, load_item(&p.blocks[b].item, 0), rb, x - b * p.pre.n_kv_heads, lds);
}

template <int D>
void launch_shared_t(const SharedParams &p, hipStream_t st) {
  const dim3 grid((unsigned)(p.unit_wgs + (int64_t)p.n_blocks * p.pre.n_kv_heads)), block(kThreads);
  // K and V of a block that no other reads need not stay in the caches
  if (p.pre.max_rows <= kRows<false>)
    hipLaunchKernelGGL((link_shared_kernel<D, false, 2>), grid, block, 0, st, p);
  else if (p.pre.nrb == 1)
    hipLaunchKernelGGL((link_shared_kernel<D, true, 2>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((link_shared_kernel<D, true, 0>), grid, block, 0, st, p);
}

}  // namespace

int shared_rows_per_block(int max_rows) { return max_rows > kRows<false> ? kRows<true> : kRows<false>; }
int shared_waves() { return kWaves; }

hipError_t launch_link_shared(const SharedParams &p, hipStream_t st) {
  if (p.unit_wgs + p.n_blocks == 0) return hipSuccess;
  if (p.pre.d_k == 128)
    launch_shared_t<128>(p, st);
  else
    launch_shared_t<64>(p, st);
  return hipGetLastError();
}

}  // namespace pic
