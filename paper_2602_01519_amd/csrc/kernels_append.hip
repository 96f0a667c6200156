// New tokens appended to growing chunks, their keys (and the step's queries) turned by their
// positions on the way, and rows taken back.
//
//   K row of token t   y_a = c x_a - s x_b,  y_b = s x_a + c x_b,  (c, s) = mag (cos, sin)(pos_t f_i)
//   V column of t      as it is, across the panels of 32 tokens that the link kernels read
//
// Bound by the bytes (each element read once and written once), for a decode step by one chain
// of loads. A launch has two kinds of workgroups. Row workgroups take a few tokens of one piece,
// form their (c, s) once and pass every query and key head over them (as rope_kernel does). Tile
// workgroups take a page (64 tokens) x 64 value dims of one head: a value row spreads over 64
// panel rows, 64 bytes apart, so whole pages go through LDS and leave as 16-byte pieces of 8
// (fp32: 4) tokens; where a group of those is only partly new, its elements go one by one. A
// page that the append begins is written to its end, zeros past the last token, so that no
// kernel meets what the page held before (0 x NaN is NaN in a product with hidden values).
//
// The pieces (a chunk's new rows within one run of pages) travel as kernel arguments: no table
// is copied, the call is one launch for up to kAppendPieces of them.
#include <algorithm>

#include "pic_internal.hpp"
#include "rope_row.hpp"

namespace pic {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 2;         // rows whose loads a lane has in flight

// 16 bytes at any address that is aligned to its elements
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

// Index of the last piece whose first unit is at most x: all pieces alike, or a search.
template <typename F>
__device__ __forceinline__ int piece_of(int x, int each, int n, F first) {
  if (each > 0) return x / each;
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first(mid) <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <typename T, bool kHalf>
__device__ __forceinline__ void append_rows(const AppendParams &p, int block, float *trig) {
  constexpr int N = Vec<T>::n;
  const int half = p.rot / 2, part = (half + 7) / 8 * 8;
  const int g = block / p.parts;
  const int u = piece_of(g, p.groups_each, p.n_pieces, [&](int i) { return p.piece[i].group0; });
  const AppendPiece &P = p.piece[u];
  const int tok0 = (g - P.group0) * p.tokens;          // within the piece
  const int ntok = min(p.tokens, P.n - tok0);
  const int slot = div_small(threadIdx.x, p.inv_lanes), chunk = threadIdx.x - slot * p.lanes;
  const RowPiece pc = row_piece<T, kHalf>(chunk, p.rot_chunks, p.d_k, p.rot_at, p.rot);
  const bool whole = pc.len >= N;
  const int h0 = (block - g * p.parts) * p.heads_per_block;
  const int heads = min(p.heads_per_block, p.q_heads + p.heads - h0);
  const float inv_heads = 1.f / (float)heads;
  const int rows = slot < p.slots ? ntok * heads : 0;
  const int64_t src0 = P.src0 + tok0;
  const int row0 = P.row0 + tok0;

  uint4 a[kBatch], b[kBatch];
  const T *src[kBatch];
  T *dst[kBatch];
  int tok[kBatch];
  const auto load = [&](int r0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + k * p.slots;
      src[k] = nullptr;
      if (r >= rows) continue;
      const int t = div_small(r, inv_heads), h = h0 + r - t * heads;
      tok[k] = t;
      if (h < p.q_heads) {
        src[k] = (const T *)p.q + (src0 + t) * p.q_stride + h * p.d_k + pc.at;
        dst[k] = (T *)p.q_out + (src0 + t) * p.q_out_stride + h * p.d_k + pc.at;
      } else {
        const int hk = h - p.q_heads;
        src[k] = (const T *)p.k + (src0 + t) * p.k_stride + hk * p.d_k + pc.at;
        dst[k] = (T *)P.k + ((int64_t)hk * P.lp + row0 + t) * p.d_k + pc.at;
      }
      if (whole) {
        a[k] = load_nt(src[k]);
        if (kHalf && pc.rot) b[k] = load_nt(src[k] + half);
      }
    }
  };
  // On their way while the angles are formed: 2000 tokens of 16 query heads and a latent row of 576,
  // one wave of workgroups, 19.8 -> 17.3 us.
  load(slot);

  for (int i = threadIdx.x; i < ntok * half; i += kThreads) {
    const int t = div_small(i, p.inv_half), j = i - t * half;
    const double rev = (double)p.positions[src0 + t] * p.rev[j];
    float s, c;
    sincospif(2.f * (float)(rev - rint(rev)), &s, &c);
    trig[t * 2 * part + j] = c * p.magnitude;
    trig[t * 2 * part + part + j] = s * p.magnitude;
  }
  __syncthreads();

  for (int r0 = slot; r0 < rows; r0 += kBatch * p.slots) {
    if (r0 != slot) load(r0);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (!src[k]) continue;
      if (pc.rot) {
        const float *cs = trig + tok[k] * 2 * part + pc.pair0;
        turn_piece<T, kHalf>(pc, src[k], dst[k], a[k], b[k], half, cs, cs + part);
      } else if (dst[k] != src[k]) {       // (queries in place: nothing to copy)
        if (whole)
          *(uint4 *)dst[k] = a[k];
        else
          for (int i = 0; i < pc.len; ++i) dst[k][i] = src[k][i];
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ void append_tile(const AppendParams &p, int block, T *tile) {
  constexpr int N = Vec<T>::n;
  constexpr int ROW = 64 + N;                // padded LDS row (elements)
  const int per_page = p.v_heads * p.v_parts;
  const int pg = block / per_page, rem = block - pg * per_page;
  const int h = rem / p.v_parts, e0 = (rem - h * p.v_parts) * 64;
  const int u = piece_of(pg, p.pages_each, p.n_pieces, [&](int i) { return p.piece[i].page0; });
  const AppendPiece &P = p.piece[u];
  const int first = (P.row0 / kTile + pg - P.page0) * kTile;   // the page's first row
  const int lo = max(P.row0, first), hi = min(P.row0 + P.n, first + kTile);
  const bool fresh = lo == first;
  const int end = fresh ? first + kTile : hi;                  // rows lo .. end are written
  if (fresh && hi < end && e0 == 0) {                          // keys past the last token
    const int per = p.d_k / N, n = (end - hi) * per;
    for (int i = threadIdx.x; i < n; i += kThreads)
      *(uint4 *)((T *)P.k + ((int64_t)h * P.lp + hi) * p.d_k + i * N) = make_uint4(0, 0, 0, 0);
  }
  if (!p.v) return;
  const int g0 = (lo - first) / N, g1 = (end - first + N - 1) / N;   // groups of N tokens
  for (int i = threadIdx.x; i < (g1 - g0) * N * (64 / N); i += kThreads) {
    const int tl = g0 * N + i / (64 / N), e = e0 + i % (64 / N) * N;
    const int row = first + tl;
    u32x4u v = {0, 0, 0, 0};
    if (row >= lo && row < hi && e < p.d_v)
      v = *(const u32x4u *)((const T *)p.v + (int64_t)(P.src0 + row - P.row0) * p.v_stride + h * p.d_v + e);
    *(uint4 *)(tile + tl * ROW + i % (64 / N) * N) = make_uint4(v.x, v.y, v.z, v.w);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * (g1 - g0); i += kThreads) {
    const int el = i / (g1 - g0), tc = g0 + i - el * (g1 - g0);
    const int e = e0 + el;
    if (e >= p.d_v) continue;
    union {
      uint4 u;
      T e[N];
    } x;
#pragma unroll
    for (int k = 0; k < N; ++k) x.e[k] = tile[(tc * N + k) * ROW + el];
    // (N tokens never straddle a panel)
    const int row = first + tc * N;
    T *dst = (T *)P.v + vt_offset(h, e, row, P.lp, p.d_v);
    if (row >= lo && row + N <= end) {
      *(uint4 *)dst = x.u;
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (row + k >= lo && row + k < end) dst[k] = x.e[k];
    }
  }
}

template <typename T, bool kHalf>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p) {
  extern __shared__ __attribute__((aligned(16))) char lds[];   // the tile, or the tokens' (c, s)
  const int rows = p.groups * p.parts;
  if ((int)blockIdx.x < rows)
    append_rows<T, kHalf>(p, blockIdx.x, (float *)lds);
  else
    append_tile<T>(p, blockIdx.x - rows, (T *)lds);
}

// Rows row0 .. row0 + n of a page to zeros, every layer: one piece and head a workgroup.
template <typename T>
__global__ __launch_bounds__(64) void clear_rows_kernel(ClearParams p) {
  const ClearPiece P = p.piece[blockIdx.x];
  const int h = blockIdx.y;
  T *k = (T *)(P.k + blockIdx.z * p.layer_bytes) + ((int64_t)h * P.lp + P.row0) * p.d_k;
  constexpr int N = Vec<T>::n;
  for (int i = threadIdx.x; i < P.n * (p.d_k / N); i += 64) *(uint4 *)(k + i * N) = make_uint4(0, 0, 0, 0);
  if (!P.v) return;
  T *v = (T *)(P.v + blockIdx.z * p.layer_bytes);
  for (int i = threadIdx.x; i < P.n * p.d_v; i += 64) {
    const int e = i / P.n, r = P.row0 + i - e * P.n;
    v[vt_offset(h, e, r, P.lp, p.d_v)] = 0;
  }
}

}  // namespace

hipError_t launch_append(AppendParams p, int esz, bool half, const DevShape &ds, hipStream_t st) {
  const int n = 16 / esz, total_heads = p.q_heads + p.heads;
  p.rot_chunks = rot_pieces(n, half, p.rot);
  p.lanes = p.rot_chunks + copy_pieces(n, p.d_k, p.rot_at, p.rot);
  p.slots = kThreads / p.lanes;
  p.inv_lanes = 1.f / (float)p.lanes;
  p.inv_half = p.rot > 0 ? 2.f / (float)p.rot : 1.f;
  int64_t tokens = 0;
  for (int i = 0; i < p.n_pieces; ++i) tokens += p.piece[i].n;
  // (tokens of a workgroup and the sharing out of their heads: as launch_rope)
  const int want = 4 * ds.cus;
  p.tokens = std::max(1, std::min(8, p.slots / total_heads));
  while (p.tokens > 1 && tokens / p.tokens < want) --p.tokens;
  p.groups = 0;
  int pages = 0;
  p.groups_each = p.pages_each = -1;
  for (int i = 0; i < p.n_pieces; ++i) {
    AppendPiece &P = p.piece[i];
    const int g = (P.n + p.tokens - 1) / p.tokens;
    const int q = (P.row0 + P.n + kTile - 1) / kTile - P.row0 / kTile;
    P.group0 = p.groups;
    P.page0 = pages;
    p.groups_each = p.groups_each == -1 || p.groups_each == g ? g : 0;
    p.pages_each = p.pages_each == -1 || p.pages_each == q ? q : 0;
    p.groups += g;
    pages += q;
  }
  p.parts = 1;
  if (p.groups < want) {
    const int most = (total_heads + p.slots - 1) / p.slots;
    p.parts = std::min(most, (want + p.groups - 1) / p.groups);
  }
  p.heads_per_block = (total_heads + p.parts - 1) / p.parts;
  p.parts = (total_heads + p.heads_per_block - 1) / p.heads_per_block;
  p.v_heads = p.heads;
  p.v_parts = p.v ? (p.d_v + 63) / 64 : 1;
  const size_t lds = std::max((size_t)p.tokens * 2 * ((p.rot / 2 + 7) / 8 * 8) * sizeof(float),
                              (size_t)64 * (64 + n) * esz);
  const dim3 grid((unsigned)(p.groups * p.parts + pages * p.v_heads * p.v_parts));
  if (esz == 4) {
    if (half)
      hipLaunchKernelGGL((append_kernel<float, true>), grid, dim3(kThreads), lds, st, p);
    else
      hipLaunchKernelGGL((append_kernel<float, false>), grid, dim3(kThreads), lds, st, p);
  } else {
    if (half)
      hipLaunchKernelGGL((append_kernel<uint16_t, true>), grid, dim3(kThreads), lds, st, p);
    else
      hipLaunchKernelGGL((append_kernel<uint16_t, false>), grid, dim3(kThreads), lds, st, p);
  }
  return hipGetLastError();
}

hipError_t launch_clear_rows(const ClearParams &p, int32_t n, int32_t n_layers, int esz, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const dim3 grid((unsigned)n, (unsigned)p.heads, (unsigned)n_layers);
  if (esz == 4)
    hipLaunchKernelGGL(clear_rows_kernel<float>, grid, dim3(64), 0, st, p);
  else
    hipLaunchKernelGGL(clear_rows_kernel<uint16_t>, grid, dim3(64), 0, st, p);
  return hipGetLastError();
}

}  // namespace pic
