// Kernels of the 4-bit chunk store: put (rounds a chunk's rows into tiles),
// single rows, copies of pages, and the read-back of the values.
//
// All are bound by the bytes they move. A workgroup of the put takes one tile
// (64 tokens of one head), four lanes to a block of 32: 16-byte reads of
// whole rows, the block's maximum by two lane exchanges, codes into an LDS
// image of the tile, which leaves in 16-byte pieces. (Tile bytes written straight
// from the registers would be 2 and 4 bytes wide for V, whose tile order runs
// across the rows.) What is read or written once passes the caches by: 7000 tokens x 8
// heads x 128 in 8 layers (229 MB in, 61 MB out) take 50 us, 5.8 TB/s, against 74 us
// with plain loads.
#include "fp4.hpp"

namespace pic {
namespace {

__device__ __forceinline__ uint4 load_once(const void *p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = __builtin_nontemporal_load((const u32x4 *)p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void store_once(void *p, uint4 v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, (u32x4 *)p);
}
__device__ __forceinline__ uint32_t pk_abs_max(uint4 x) {
  auto hi = [](uint32_t a, uint32_t b) {
    a &= 0x7fff7fffu;
    b &= 0x7fff7fffu;
    const uint32_t lo = max(a & 0xffffu, b & 0xffffu), up = max(a >> 16, b >> 16);
    return lo | up << 16;
  };
  const uint32_t m = hi(hi(x.x, x.y), hi(x.z, x.w));
  return max(m & 0xffffu, m >> 16);
}
// Largest over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));
}

// Stores the 8 codes of elements e .. e + 7 of a key into a tile (LDS or
// global memory) and, from the first lane of the block, its scale.
template <int D>
__device__ __forceinline__ void store8(char *tile, bool v, int key, int e, uint32_t code,
                                       uint32_t scale) {
  typedef Fp4Tile<D> T;
  if (!v) {
    *(uint32_t *)(tile + T::k_code(key, e)) = code;
  } else if (D == 128) {
    *(uint32_t *)(tile + T::v_code(key, e)) = code;
  } else {
    *(uint16_t *)(tile + T::v_code(key, e)) = (uint16_t)code;
    *(uint16_t *)(tile + T::v_code(key, e + 4)) = (uint16_t)(code >> 16);
  }
  if (e % 32 == 0) tile[v ? T::v_scale(key, e / 32) : T::k_scale(key, e / 32)] = (char)scale;
}

// grid: (pages of the run, heads, layers)
template <int D>
__global__ __launch_bounds__(256) void fp4_put_kernel(Fp4Put p) {
  typedef Fp4Tile<D> T;
  __shared__ uint4 tile[T::kBytes / 16];
  constexpr int kPer = D / 8;                       // lanes of a row
  constexpr int kIter = 64 * kPer / 256;
  const int h = blockIdx.y, tok0 = blockIdx.x * 64;
  const int64_t src = (int64_t)blockIdx.z * p.src_layer;
  const int e = threadIdx.x % kPer * 8;
  uint4 x[2][kIter];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int j = 0; j < kIter; ++j) {
      const int key = threadIdx.x / kPer + j * (256 / kPer);
      x[kv][j] = make_uint4(0, 0, 0, 0);            // rows past the last: zeros
      if (tok0 + key < p.n_tokens)
        x[kv][j] = load_once((kv ? p.v : p.k) + src + ((int64_t)(tok0 + key) * p.heads + h) * D + e);
    }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int j = 0; j < kIter; ++j) {
      const uint32_t s = fp4_scale_byte(quad_max(pk_abs_max(x[kv][j])));
      store8<D>((char *)tile, kv, threadIdx.x / kPer + j * (256 / kPer), e,
                fp4_encode8(x[kv][j], fp4_scale(s)), s);
    }
  __syncthreads();
  uint4 *dst = (uint4 *)(p.dst + (int64_t)blockIdx.z * p.layer_bytes +
                         ((int64_t)blockIdx.x * p.heads + h) * T::kBytes);
  for (int i = threadIdx.x; i < T::kBytes / 16; i += 256) dst[i] = tile[i];
}

// grid: (blocks of rows x heads); rows of one layer into a derived chunk.
template <int D, int kRows>
__global__ __launch_bounds__(256) void fp4_write_rows_kernel(WriteRows<kRows> w, const uint16_t *k,
                                                             const uint16_t *v, int n, int heads) {
  constexpr int kPer = D / 8;
  const int64_t task = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int e = (int)(task % kPer) * 8;
  const int64_t row = task / kPer;                  // (row of the list, head)
  const int h = (int)(row % heads);
  const int i = (int)(row / heads);
  // lanes of a quad share their row, so that they stay together
  if (i >= n) return;
  const int tok = w.row[i];
  int vi = 0;
  while (vi + 1 < w.n_views && tok >= w.view[vi + 1].tok0) ++vi;
  const int t = tok - w.view[vi].tok0;
  char *tile = (char *)w.view[vi].k + ((int64_t)(t / 64) * heads + h) * Fp4Tile<D>::kBytes;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const uint4 x = *(const uint4 *)((kv ? v : k) + row * D + e);
    const uint32_t s = fp4_scale_byte(quad_max(pk_abs_max(x)));
    store8<D>(tile, kv, t % 64, e, fp4_encode8(x, fp4_scale(s)), s);
  }
}

// grid: (16-byte units of a page / 256, pages, layers)
__global__ __launch_bounds__(256) void fp4_copy_pages_kernel(PageCopies c, int64_t page_bytes) {
  const PageCopy &pg = c.page[blockIdx.y];
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16;
  if (at >= page_bytes) return;
  const int64_t off = (int64_t)blockIdx.z * c.layer_bytes + at;
  *(uint4 *)(pg.dst_k + off) = *(const uint4 *)(pg.src_k + off);
}

struct GatherLinks {
  int32_t n;
  int32_t tile0[kGatherLinks];      // the link's first workgroup
  const char *page[kGatherLinks];
  int32_t len[kGatherLinks], tok0[kGatherLinks];
};

// Values of the linked rows, token-major bf16. grid: (tiles, heads)
template <int D>
__global__ __launch_bounds__(256) void fp4_gather_kernel(GatherLinks links, int heads, uint16_t *k,
                                                         uint16_t *v) {
  typedef Fp4Tile<D> T;
  __shared__ uint4 tile[T::kBytes / 16];
  int li = 0;
  while (li + 1 < links.n && (int)blockIdx.x >= links.tile0[li + 1]) ++li;
  struct {
    const char *k;
    int32_t len, tok0;
  } const L{links.page[li], links.len[li], links.tok0[li]};
  const int t = blockIdx.x - links.tile0[li], h = blockIdx.y;
  const uint4 *src = (const uint4 *)(L.k + ((int64_t)t * heads + h) * T::kBytes);
  for (int i = threadIdx.x; i < T::kBytes / 16; i += 256) tile[i] = src[i];
  __syncthreads();
  const char *b = (const char *)tile;
  constexpr int kPer = D / 8;
  const int e = threadIdx.x % kPer * 8;
#pragma unroll
  for (int j = 0; j < 64 * kPer / 256; ++j) {
    const int key = threadIdx.x / kPer + j * (256 / kPer);
    if (t * 64 + key >= L.len) continue;
    const int64_t out = ((int64_t)(L.tok0 + t * 64 + key) * heads + h) * D + e;
    const float ks = fp4_scale((uint8_t)b[T::k_scale(key, e / 32)]);
    const float vs = fp4_scale((uint8_t)b[T::v_scale(key, e / 32)]);
    const uint32_t kc = *(const uint32_t *)(b + T::k_code(key, e));
    uint32_t vc;
    if (D == 128)
      vc = *(const uint32_t *)(b + T::v_code(key, e));
    else
      vc = *(const uint16_t *)(b + T::v_code(key, e)) |
           (uint32_t)*(const uint16_t *)(b + T::v_code(key, e + 4)) << 16;
    store_once(k + out, fp4_decode8(kc, ks));
    store_once(v + out, fp4_decode8(vc, vs));
  }
}

template <int kRows>
hipError_t write_rows(const RowView *views, int32_t n_views, const int32_t *rows, int32_t n,
                      const void *k, const void *v, int32_t heads, int32_t d, hipStream_t st) {
  WriteRows<kRows> w{};
  for (int i = 0; i < n_views; ++i) w.view[i] = views[i];
  w.n_views = n_views;
  for (int i = 0; i < n; ++i) w.row[i] = rows[i];
  const int64_t tasks = (int64_t)n * heads * (d / 8);
  const dim3 grid((unsigned)((tasks + 255) / 256));
  if (d == 128)
    hipLaunchKernelGGL((fp4_write_rows_kernel<128, kRows>), grid, dim3(256), 0, st, w,
                       (const uint16_t *)k, (const uint16_t *)v, n, heads);
  else
    hipLaunchKernelGGL((fp4_write_rows_kernel<64, kRows>), grid, dim3(256), 0, st, w,
                       (const uint16_t *)k, (const uint16_t *)v, n, heads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp4_put(const Fp4Put &p, int32_t d, int32_t n_layers, hipStream_t st) {
  const dim3 grid((unsigned)((p.n_tokens + 63) / 64), (unsigned)p.heads, (unsigned)n_layers);
  if (d == 128)
    hipLaunchKernelGGL(fp4_put_kernel<128>, grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(fp4_put_kernel<64>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_fp4_write_rows(const RowView *views, int32_t n_views, const int32_t *rows,
                                 int32_t n, const void *k, const void *v, int32_t heads, int32_t d,
                                 hipStream_t st) {
  return n <= kWriteRowsFew ? write_rows<kWriteRowsFew>(views, n_views, rows, n, k, v, heads, d, st)
                            : write_rows<kWriteRowsMost>(views, n_views, rows, n, k, v, heads, d, st);
}

hipError_t launch_fp4_copy_pages(const PageCopies &c, int32_t n, int32_t n_layers, hipStream_t st) {
  const int64_t bytes = fp4_page_bytes(c.heads, c.d_k);
  const dim3 grid((unsigned)((bytes / 16 + 255) / 256), (unsigned)n, (unsigned)n_layers);
  hipLaunchKernelGGL(fp4_copy_pages_kernel, grid, dim3(256), 0, st, c, bytes);
  return hipGetLastError();
}

hipError_t launch_fp4_gather(const LinkEntry *links, int32_t n_links, int32_t heads, int32_t d,
                             void *k, void *v, hipStream_t st) {
  GatherLinks g{};
  g.n = n_links;
  int32_t tiles = 0;
  for (int32_t i = 0; i < n_links; ++i) {
    g.tile0[i] = tiles;
    g.page[i] = (const char *)links[i].k;
    g.len[i] = links[i].len;
    g.tok0[i] = links[i].tok0;
    tiles += (links[i].len + 63) / 64;
  }
  const dim3 grid((unsigned)tiles, (unsigned)heads);
  if (d == 128)
    hipLaunchKernelGGL(fp4_gather_kernel<128>, grid, dim3(256), 0, st, g, heads, (uint16_t *)k,
                       (uint16_t *)v);
  else
    hipLaunchKernelGGL(fp4_gather_kernel<64>, grid, dim3(256), 0, st, g, heads, (uint16_t *)k,
                       (uint16_t *)v);
  return hipGetLastError();
}

}  // namespace pic
