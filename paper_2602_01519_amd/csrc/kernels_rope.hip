// Rotary positions: pairs of a head's elements turned by position * frequency,
// forward and transposed, for up to kRopeTensors tensors that share their
// positions (a layer's queries and keys) in one launch.
//
//   y_a = c x_a - s x_b,  y_b = s x_a + c x_b,  (c, s) = mag (cos, sin)(pos f_i)
//   transposed: s -> -s (the gradient of the forward map)
//
// Bound by the bytes: every element is read and written once. A workgroup
// takes a few tokens: it forms their (c, s) once, in LDS, and passes them to all
// heads. The angle is held in revolutions in 64 bits, t = pos f / (2 pi), and
// reduced there (t - rint t, exact), so that far positions lose nothing: at
// 2^31 the product's rounding is 2^-24 revolutions. Sine and cosine are then
// fp32 of at most half a turn. Products in fp32, one rounding to the output.
// 8192 tokens x (32 + 8) heads x 128, bf16, slices of one projection: 29.6 us, 5.7 TB/s of a
// copy's 4.7; 4099 x 17 x 192 fp32, 64 of them turned: 25.8 us, 4.2 TB/s. (The first rows'
// loads before the angles: 34 and 24.4 us. At most 64 registers, eight waves per
// SIMD: the latter 27.1 us without.)
//
// A row's elements are cut into chunks of 16 bytes, a lane each: kRot chunks
// hold rotated pairs (half layout: two pieces, one from each half), the others
// are copied (out of place only; in place they are not touched). A chunk that
// the part's end cuts short goes element by element, which keeps every size on
// the same path.
#include <algorithm>

#include "pic_internal.hpp"

namespace pic {
namespace {

constexpr int kThreads = 256;
constexpr int kMostBlocks = (1 << 24) - 1;     // of kThreads in one launch
constexpr int kBatch = 2;         // rows whose loads a lane has in flight

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

template <typename T, bool kHalf>
__global__ __launch_bounds__(kThreads, 8) void rope_kernel(RopeParams p) {
  typedef Vec<T> V;
  constexpr int N = V::n;
  extern __shared__ float trig[];     // [token][cos: half][sin: half], each part 16-byte aligned
  const int half = p.rot / 2, part = (half + 7) / 8 * 8;
  const int tok0 = blockIdx.x * p.tokens;
  const int ntok = min(p.tokens, p.n_tokens - tok0);
  const int slot = div_small(threadIdx.x, p.inv_lanes), chunk = threadIdx.x - slot * p.lanes;
  // this lane's piece of a row
  const bool rot = chunk < p.rot_chunks;
  int at, len;                        // first element; elements up to the part's end
  if (rot) {
    at = p.rot_at + chunk * N;
    len = (kHalf ? half : p.rot) - chunk * N;
  } else {
    const int c = chunk - p.rot_chunks, lead = (p.rot_at + N - 1) / N;
    at = c < lead ? c * N : p.rot_at + p.rot + (c - lead) * N;
    len = (c < lead ? p.rot_at : p.width) - at;
  }
  const bool whole = len >= N;
  const int pair0 = kHalf ? chunk * N : chunk * N / 2;
  const int h0 = blockIdx.y * p.heads_per_block;
  const int heads = min(p.heads_per_block, p.heads - h0);
  const float inv_heads = 1.f / (float)heads;
  const int rows = slot < p.slots ? ntok * heads : 0;

  uint4 a[kBatch], b[kBatch];
  const T *src[kBatch];
  T *dst[kBatch];
  int tok[kBatch];
  auto load = [&](int r0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + k * p.slots;
      src[k] = nullptr;
      if (r >= rows) continue;
      const int t = div_small(r, inv_heads);
      int h = h0 + r - t * heads;
      tok[k] = t;
      int i = 0;
      while (h >= p.t[i].heads) h -= p.t[i++].heads;
      src[k] = (const T *)p.t[i].x + (tok0 + t) * p.t[i].x_stride + h * p.width + at;
      dst[k] = (T *)p.t[i].out + (tok0 + t) * p.t[i].out_stride + h * p.width + at;
      if (whole) {
        a[k] = load_nt(src[k]);
        if (kHalf && rot) b[k] = load_nt(src[k] + half);
      }
    }
  };
  for (int i = threadIdx.x; i < ntok * half; i += kThreads) {
    const int t = div_small(i, p.inv_half), j = i - t * half;
    const double rev = (double)p.positions[tok0 + t] * p.rev[j];
    float s, c;
    sincospif(2.f * (float)(rev - rint(rev)), &s, &c);
    trig[t * 2 * part + j] = c * p.magnitude;
    trig[t * 2 * part + part + j] = s * p.sine;
  }
  __syncthreads();

  for (int r0 = slot; r0 < rows; r0 += kBatch * p.slots) {
    load(r0);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (!src[k]) continue;
      if (!rot) {
        if (dst[k] == src[k]) continue;      // in place beside an out-of-place tensor
        if (whole) {
          *(uint4 *)dst[k] = a[k];
        } else {
          for (int i = 0; i < len; ++i) dst[k][i] = src[k][i];
        }
        continue;
      }
      const float *cs = trig + tok[k] * 2 * part + pair0, *sn = cs + part;
      if (whole) {
        float x[N], y[N];
        if (kHalf) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float u = V::get(a[k], i), w = V::get(b[k], i), c = cs[i], s = sn[i];
            x[i] = u * c - w * s;
            y[i] = u * s + w * c;
          }
          *(uint4 *)dst[k] = V::put(x);
          *(uint4 *)(dst[k] + half) = V::put(y);
        } else {
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const float u = V::get(a[k], i), w = V::get(a[k], i + 1), c = cs[i / 2], s = sn[i / 2];
            x[i] = u * c - w * s;
            x[i + 1] = u * s + w * c;
          }
          *(uint4 *)dst[k] = V::put(x);
        }
      } else {
        const int step = kHalf ? 1 : 2, other = kHalf ? half : 1;
        for (int i = 0; i < len; i += step) {
          const float u = V::load(src[k] + i), w = V::load(src[k] + i + other);
          const float c = cs[i / step], s = sn[i / step];
          V::store(dst[k] + i, u * c - w * s);
          V::store(dst[k] + i + other, u * s + w * c);
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(RopeParams p, int dtype, bool half, const DevShape &ds, hipStream_t st) {
  const int n = dtype == 0 ? 4 : 8;
  p.rot_chunks = (half ? p.rot / 2 + n - 1 : p.rot + n - 1) / n;
  // copies only where some tensor is not in place
  int copies = 0;
  for (int i = 0; i < p.n_tensors; ++i)
    if (p.t[i].x != p.t[i].out) copies = (p.rot_at + n - 1) / n + (p.width - p.rot_at - p.rot + n - 1) / n;
  p.lanes = p.rot_chunks + copies;
  p.slots = kThreads / p.lanes;
  p.inv_lanes = 1.f / (float)p.lanes;
  p.inv_half = 1.f / (float)(p.rot / 2);
  // Tokens of a workgroup: one pass of its lanes over all heads, one to eight (many
  // small workgroups: the angles of some are formed under the loads of others; 8192 tokens
  // x 40 heads, 1 / 2 / 4 / 8 tokens: 36.5 / 37.9 / 41.6 / 41.9 us). Where that
  // leaves fewer than four workgroups per CU, single tokens, and their heads shared
  // out, down to one pass.
  const int want = 4 * ds.cus;
  p.tokens = p.slots / p.heads < 1 ? 1 : p.slots / p.heads > 8 ? 8 : p.slots / p.heads;
  while (p.tokens > 1 && p.n_tokens / p.tokens < want) --p.tokens;
  const int64_t blocks = ((int64_t)p.n_tokens + p.tokens - 1) / p.tokens;
  int parts = 1;
  if (blocks < want) {
    const int most = (p.heads + p.slots - 1) / p.slots;
    parts = (int)((want + blocks - 1) / blocks);
    if (parts > most) parts = most;
  }
  p.heads_per_block = (p.heads + parts - 1) / parts;
  const size_t lds = (size_t)p.tokens * 2 * ((p.rot / 2 + 7) / 8 * 8) * sizeof(float);
  // One launch but for very many tokens (2^24 workgroups or more): a launch's threads are
  // counted in 32 bits, and what lies above is dropped without an error.
  const int64_t all = p.n_tokens, most = (int64_t)kMostBlocks * p.tokens;
  const int esz = dtype == 0 ? 4 : 2;
  for (int64_t at = 0; at < all; at += most) {
    p.n_tokens = (int32_t)std::min(all - at, most);
    const dim3 grid((unsigned)((p.n_tokens + (int64_t)p.tokens - 1) / p.tokens),
                    (unsigned)((p.heads + p.heads_per_block - 1) / p.heads_per_block));
    if (dtype == 0) {
      if (half)
        hipLaunchKernelGGL((rope_kernel<float, true>), grid, dim3(kThreads), lds, st, p);
      else
        hipLaunchKernelGGL((rope_kernel<float, false>), grid, dim3(kThreads), lds, st, p);
    } else {
      if (half)
        hipLaunchKernelGGL((rope_kernel<uint16_t, true>), grid, dim3(kThreads), lds, st, p);
      else
        hipLaunchKernelGGL((rope_kernel<uint16_t, false>), grid, dim3(kThreads), lds, st, p);
    }
    p.positions += p.n_tokens;
    for (int i = 0; i < p.n_tensors; ++i) {
      p.t[i].x = (const char *)p.t[i].x + p.n_tokens * p.t[i].x_stride * esz;
      p.t[i].out = (char *)p.t[i].out + p.n_tokens * p.t[i].out_stride * esz;
    }
  }
  return hipGetLastError();
}

}  // namespace pic
