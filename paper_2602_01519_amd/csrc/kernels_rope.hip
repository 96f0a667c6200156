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
#include "rope_row.hpp"

namespace pic {
namespace {

constexpr int kThreads = 256;
constexpr int kMostBlocks = (1 << 24) - 1;     // of kThreads in one launch
constexpr int kBatch = 2;         // rows whose loads a lane has in flight

template <typename T, bool kHalf>
__global__ __launch_bounds__(kThreads, 8) void rope_kernel(RopeParams p) {
  constexpr int N = Vec<T>::n;
  extern __shared__ float trig[];     // [token][cos: half][sin: half], each part 16-byte aligned
  const int half = p.rot / 2, part = (half + 7) / 8 * 8;
  const int tok0 = blockIdx.x * p.tokens;
  const int ntok = min(p.tokens, p.n_tokens - tok0);
  const int slot = div_small(threadIdx.x, p.inv_lanes), chunk = threadIdx.x - slot * p.lanes;
  // this lane's piece of a row
  const RowPiece pc = row_piece<T, kHalf>(chunk, p.rot_chunks, p.width, p.rot_at, p.rot);
  const bool rot = pc.rot, whole = pc.len >= N;
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
      src[k] = (const T *)p.t[i].x + (tok0 + t) * p.t[i].x_stride + h * p.width + pc.at;
      dst[k] = (T *)p.t[i].out + (tok0 + t) * p.t[i].out_stride + h * p.width + pc.at;
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
          for (int i = 0; i < pc.len; ++i) dst[k][i] = src[k][i];
        }
        continue;
      }
      const float *cs = trig + tok[k] * 2 * part + pc.pair0;
      turn_piece<T, kHalf>(pc, src[k], dst[k], a[k], b[k], half, cs, cs + part);
    }
  }
}

}  // namespace

hipError_t launch_rope(RopeParams p, int dtype, bool half, const DevShape &ds, hipStream_t st) {
  const int n = dtype == 0 ? 4 : 8;
  p.rot_chunks = rot_pieces(n, half, p.rot);
  // copies only where some tensor is not in place
  int copies = 0;
  for (int i = 0; i < p.n_tensors; ++i)
    if (p.t[i].x != p.t[i].out) copies = copy_pieces(n, p.width, p.rot_at, p.rot);
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
