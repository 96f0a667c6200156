// What the kernels that turn rows by their positions share: 16-byte pieces of a row's
// elements, and the turn of one piece (see kernels_rope.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pic {

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int n = 4;
  __device__ static float get(const uint4 &v, int i) {
    return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
  }
  __device__ static uint4 put(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                      __float_as_uint(x[3]));
  }
  __device__ static float load(const float *p) { return *p; }
  __device__ static void store(float *p, float x) { *p = x; }
};
template <>
struct Vec<uint16_t> {
  static constexpr int n = 8;
  __device__ static float get(const uint4 &v, int i) {
    const uint32_t w = i / 2 == 0 ? v.x : i / 2 == 1 ? v.y : i / 2 == 2 ? v.z : v.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ static uint4 put(const float (&x)[8]) {
    __bf16 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    return __builtin_bit_cast(uint4, v);
  }
  __device__ static float load(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
  __device__ static void store(uint16_t *p, float x) {
    *p = __builtin_bit_cast(uint16_t, (__bf16)x);
  }
};

// 16 bytes read once (nontemporal: 8192 tokens x 40 heads x 128 bf16 in 32.5 us
// against 36.5).
__device__ __forceinline__ uint4 load_nt(const void *p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = __builtin_nontemporal_load((const u32x4 *)p);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// Quotient of small numbers (below 2^22) by a constant's reciprocal.
__device__ __forceinline__ int div_small(int x, float inv) { return (int)(((float)x + 0.5f) * inv); }

// A lane's piece of a row: 16 bytes at element `at`, fewer where the part ends; for
// the half layout also those half a rotated part further on.
struct RowPiece {
  bool rot;             // rotated pairs (else copied)
  int at, len;          // first element; elements up to the part's end
  int pair0;            // first pair
};
// Piece `chunk` of a row: the rotated part's rot_chunks first, then the copied ones.
template <typename T, bool kHalf>
__device__ __forceinline__ RowPiece row_piece(int chunk, int rot_chunks, int width, int rot_at, int rot) {
  constexpr int N = Vec<T>::n;
  RowPiece r;
  r.rot = chunk < rot_chunks;
  if (r.rot) {
    r.at = rot_at + chunk * N;
    r.len = (kHalf ? rot / 2 : rot) - chunk * N;
  } else {
    const int c = chunk - rot_chunks, lead = (rot_at + N - 1) / N;
    r.at = c < lead ? c * N : rot_at + rot + (c - lead) * N;
    r.len = (c < lead ? rot_at : width) - r.at;
  }
  r.pair0 = kHalf ? chunk * N : chunk * N / 2;
  return r;
}
// Pieces of a row's rotated part, and of the others.
inline int rot_pieces(int n, bool half, int rot) { return half ? (rot / 2 + n - 1) / n : (rot + n - 1) / n; }
inline int copy_pieces(int n, int width, int rot_at, int rot) {
  return (rot_at + n - 1) / n + (width - rot_at - rot + n - 1) / n;
}

// Writes a piece, turned: src, dst at its first element; a, b its 16 bytes (and those
// `half` on) where it is whole; cs, sn: cos and sin of its pairs.
template <typename T, bool kHalf>
__device__ __forceinline__ void turn_piece(const RowPiece &pc, const T *src, T *dst, const uint4 &a,
                                           const uint4 &b, int half, const float *cs, const float *sn) {
  typedef Vec<T> V;
  constexpr int N = V::n;
  if (pc.len >= N) {
    float x[N], y[N];
    if (kHalf) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float u = V::get(a, i), w = V::get(b, i), c = cs[i], s = sn[i];
        x[i] = u * c - w * s;
        y[i] = u * s + w * c;
      }
      *(uint4 *)dst = V::put(x);
      *(uint4 *)(dst + half) = V::put(y);
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float u = V::get(a, i), w = V::get(a, i + 1), c = cs[i / 2], s = sn[i / 2];
        x[i] = u * c - w * s;
        x[i + 1] = u * s + w * c;
      }
      *(uint4 *)dst = V::put(x);
    }
    return;
  }
  const int step = kHalf ? 1 : 2, other = kHalf ? half : 1;
  for (int i = 0; i < pc.len; i += step) {
    const float u = V::load(src + i), w = V::load(src + i + other);
    const float c = cs[i / step], s = sn[i / step];
    V::store(dst + i, u * c - w * s);
    V::store(dst + i + other, u * s + w * c);
  }
}

}  // namespace pic
