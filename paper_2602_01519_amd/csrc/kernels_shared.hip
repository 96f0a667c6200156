// Link attention of requests that share linked chunks: the partial softmax states of a row, those
// over the rows that its group shares and those over its request's own, merged.
//
//   M = max m_i,  L = sum l_i 2^(m_i - M),  out = sum o_i 2^(m_i - M) / L,  lse = ln(2^M L)
//
// Bound by the partials' bytes, for few rows by latency: as in combine_kernel, kLanes lanes take
// a row (16, 32 or 64: d_v up to 64, 128, more), kGpr groups of them share a row's pieces where
// these are many, and a group has kB pieces' loads in flight.
#include <algorithm>
#include <cfloat>

#include "pic_internal.hpp"

namespace pic {
namespace {

__device__ __forceinline__ float largest(float4 v) {     // NaN if one is
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(v.x), fabsf(v.y)),
                                       __builtin_elementwise_maximum(fabsf(v.z), fabsf(v.w)));
}
__device__ __forceinline__ void store_quad(float *out, float4 v) { *(float4 *)out = v; }
__device__ __forceinline__ void store_quad(uint16_t *out, float4 v) {
  const __bf16 x[4] = {(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
  *(uint2 *)out = __builtin_bit_cast(uint2, x);
}
__device__ __forceinline__ void add_scaled(float4 &a, float w, const float4 &v) {
  a = make_float4(a.x + w * v.x, a.y + w * v.y, a.z + w * v.z, a.w + w * v.w);
}

constexpr int kMostBlocks = (1 << 24) - 1;     // (a launch's threads are counted in 32 bits)

template <typename T, int kLanes, int kChunks, int kGpr>
__global__ __launch_bounds__(256) void merge_kernel(MergeParams p) {
  constexpr int kB = 4;
  constexpr int kGroups = 256 / kLanes, kRows = kGroups / kGpr;
  __shared__ float4 so[kGpr > 1 ? kGroups : 1][kGpr > 1 ? kChunks * kLanes : 1];
  __shared__ float sm[kGroups], sl[kGroups];
  const int grp = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, sub = grp % kGpr;
  typedef __attribute__((address_space(4))) const MergeEntry *const_entries;
  const int r = blockIdx.x / p.blocks, b = blockIdx.x - r * p.blocks;
  MergeEntry e = p.one;
  if (p.entries) {
    const const_entries t = (const_entries)p.entries + r;
    e.row0 = t->row0;
    e.rows = t->rows;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      e.part[i] = t->part[i];
      e.stride[i] = t->stride[i];
      e.splits[i] = t->splits[i];
    }
  }
  const int nrows = e.rows;
  if (b * kRows >= nrows) return;
  const int i = b * kRows + grp / kGpr;
  const bool valid = i < nrows;
  const int sa = e.splits[0], S = valid ? sa + e.splits[1] : 0, dv = p.d_v;
  const int64_t at_a = (int64_t)e.part[0] + i, at_b = (int64_t)e.part[1] + i;
  const int64_t step_a = e.stride[0], step_b = e.stride[1];
  struct Piece {
    const float *o;
    float m, l;
  };
  auto piece = [&](int s) {
    const bool first = s < sa;
    const Partials &q = first ? p.src[0] : p.src[1];
    const int64_t pr = first ? at_a + s * step_a : at_b + (s - sa) * step_b;
    return Piece{q.o + pr * dv, q.m[pr], q.l[pr]};
  };

  float M = -INFINITY, L = 0.f;
  float4 acc[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
  auto rescale = [&](float m) {
    const float f = M == -INFINITY ? 0.f : exp2f(M - m);
    L *= f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) acc[c] = make_float4(acc[c].x * f, acc[c].y * f, acc[c].z * f, acc[c].w * f);
    M = m;
  };
  for (int s0 = sub; s0 < S; s0 += kB * kGpr) {
    Piece pc[kB];
    float4 v[kB][kChunks];
    float top = M;
#pragma unroll
    for (int k = 0; k < kB; ++k) {
      const int s = s0 + k * kGpr;
      pc[k] = piece(min(s, S - 1));
      if (s >= S) pc[k].m = -INFINITY;
      top = fmaxf(top, pc[k].m);
    }
#pragma unroll
    for (int k = 0; k < kB; ++k)
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int at = 4 * (kLanes * c + lane);
        // (with p.sparse the values of a piece that holds no key may be unwritten: they wait for
        // the maxima)
        v[k][c] = at < dv && s0 + k * kGpr < S && (!p.sparse || pc[k].m != -INFINITY)
                      ? *(const float4 *)(pc[k].o + at)
                      : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    if (top == -INFINITY) continue;
    rescale(top);
#pragma unroll
    for (int k = 0; k < kB; ++k) {
      if (pc[k].m == -INFINITY) continue;
      const float w = exp2f(pc[k].m - top);
      L += w * pc[k].l;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) add_scaled(acc[c], w, v[k][c]);
    }
  }
  if constexpr (kGpr > 1) {                 // the row's first group takes in what the others hold
    if (sub > 0) {
#pragma unroll
      for (int c = 0; c < kChunks; ++c) so[grp][kLanes * c + lane] = acc[c];
      if (lane == 0) {
        sm[grp] = M;
        sl[grp] = L;
      }
    }
    __syncthreads();
    if (sub > 0) return;
    float top = M;
#pragma unroll
    for (int k = 1; k < kGpr; ++k) top = fmaxf(top, sm[grp + k]);
    if (top != -INFINITY) {
      rescale(top);
#pragma unroll
      for (int k = 1; k < kGpr; ++k) {
        if (sm[grp + k] == -INFINITY) continue;
        const float w = exp2f(sm[grp + k] - top);
        L += w * sl[grp + k];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) add_scaled(acc[c], w, so[grp + k][kLanes * c + lane]);
      }
    }
  }
  if (!valid) return;
  const int64_t orow = (int64_t)e.row0 + i;
  T *out = (T *)p.out + orow * dv;
  const float inv = M == -INFINITY ? 0.f : 1.f / L;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int at = 4 * (kLanes * c + lane);
    if (at >= dv) continue;
    float4 a = make_float4(acc[c].x * inv, acc[c].y * inv, acc[c].z * inv, acc[c].w * inv);
    if (M != -INFINITY && !(largest(acc[c]) <= FLT_MAX)) {
      // sums of large values that pass the fp32 range before they are divided by L: again,
      // with weights that sum to one
      a = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < S; ++s) {
        const Piece x = piece(s);
        if (x.m == -INFINITY) continue;
        add_scaled(a, exp2f(x.m - M) * inv, *(const float4 *)(x.o + at));
      }
    }
    store_quad(out + at, a);
  }
  if (p.lse && lane == 0) p.lse[orow] = M == -INFINITY ? -INFINITY : log_sum(M, L);
}

template <typename T, int kLanes, int kChunks>
hipError_t launch_merge_t(MergeParams p, int32_t batch, int32_t max_rows, int32_t rows, int32_t pieces, hipStream_t st) {
  auto go = [&](auto kg) {
    constexpr int kGpr = decltype(kg)::value;
    const int per = 256 / kLanes / kGpr;
    p.blocks = (max_rows + per - 1) / per;
    const int most = std::max(1, kMostBlocks / p.blocks);
    const MergeEntry *all = p.entries;
    for (int32_t at = 0; at < batch; at += most) {
      p.entries = all ? all + at : nullptr;
      hipLaunchKernelGGL((merge_kernel<T, kLanes, kChunks, kGpr>),
                         dim3((unsigned)p.blocks * std::min(most, batch - at)), dim3(256), 0, st, p);
    }
    return hipGetLastError();
  };
  // One pass of each group over its pieces, as far as the rows leave room for it: about two
  // thousand workgroups run at once.
  const auto room = [&](int gpr) { return (int64_t)rows * kLanes * gpr <= (int64_t)256 * 2048; };
  if constexpr (kLanes < 64)
    if (pieces > 16 && room(8)) return go(std::integral_constant<int, 8>());
  if (pieces > 8 && room(4)) return go(std::integral_constant<int, 4>());
  if (pieces > 4 && room(2)) return go(std::integral_constant<int, 2>());
  return go(std::integral_constant<int, 1>());
}

template <typename T>
hipError_t launch_merge_w(const MergeParams &p, int32_t batch, int32_t max_rows, int32_t rows, int32_t pieces, hipStream_t st) {
  if (p.d_v <= 64) return launch_merge_t<T, 16, 1>(p, batch, max_rows, rows, pieces, st);
  if (p.d_v <= 128) return launch_merge_t<T, 32, 1>(p, batch, max_rows, rows, pieces, st);
  if (p.d_v <= 512) return launch_merge_t<T, 64, 2>(p, batch, max_rows, rows, pieces, st);
  return launch_merge_t<T, 64, 4>(p, batch, max_rows, rows, pieces, st);
}

}  // namespace

int merge_most_rows() { return kMostBlocks * (256 / 64); }

hipError_t launch_merge(const MergeParams &p, int dtype, int32_t batch, int32_t max_rows, int32_t rows,
                        int32_t pieces, hipStream_t st) {
  if (batch <= 0 || max_rows <= 0) return hipSuccess;
  return dtype == 0 ? launch_merge_w<float>(p, batch, max_rows, rows, pieces, st)
                    : launch_merge_w<uint16_t>(p, batch, max_rows, rows, pieces, st);
}

}  // namespace pic
