// bf16 GQA link attention for decode-shaped requests on gfx950, head dim 128.
//
// Decode reads every linked key once per query token (a generated token is a
// query token, Sec. 4), so the work is a stream over the request's
// concatenated chunk KV (Sec. 4.2) bounded by HBM bandwidth, not by math.
// Each wave owns one kv head of a work item (a piece of a request's keys) and streams its
// key range in 32-key tiles straight from HBM into registers, already in the
// operand layout of v_mfma_f32_16x16x32_bf16:
//   S^T[32 keys][16 cols] = K . Q^T    2 key blocks x 4 d steps  (8 MFMAs)
//   O^T[128][16 cols]    += V^T . P^T  8 value blocks x 1 step   (8 MFMAs)
// The 16 columns are the work item's rows (query token x GQA head, at most
// 16; unused columns are zero). The next tile's 16 x 16-byte loads per lane
// are in flight while the current tile is computed (register double
// buffering, loop unrolled by two), so each wave keeps 16 KB in flight.
//
// Row permutation: M index m of key block b reads key row 8*(m/4) + 4*b +
// m%4, so after QK^T lane l holds the scores of keys 8*(l/16) + 0..7 (four
// per block) for column l%16 -- exactly the 8 keys its PV operand needs, and
// the matching V^T operand is one 16-byte load of those 8 keys.
//
// Softmax: log2 domain, exact running max per tile (column max over the 4
// lane groups by two lane swaps), unnormalised partial (o, m, l) written per
// split and merged by the log-sum-exp combine (or normalised here when the
// range is not split).
#include "decode_d128.hpp"

namespace pic {
namespace {

constexpr int kWaves = 4;

template <bool kFull>
__global__ __launch_bounds__(256, 2) void link_decode_d128_kernel(LinkParams p) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // one (item, kv head) per wave
  const int u = blockIdx.x * kWaves + wave;
  if (u >= p.n_items * p.n_kv_heads) return;
  decode_d128::wave_unit<false, kFull>(p, u, lane, nullptr);
}

}  // namespace

int decode_d128_max_rows() { return decode_d128::kCols; }

hipError_t launch_link_decode_d128(const LinkParams &p, hipStream_t st, const char **name) {
  *name = "link_decode_d128_kernel";
  const int64_t items = (int64_t)p.n_items * p.n_kv_heads;
  dim3 grid((unsigned)((items + kWaves - 1) / kWaves));
  if (p.full_sums)
    hipLaunchKernelGGL(link_decode_d128_kernel<true>, grid, dim3(64 * kWaves), 0, st, p);
  else
    hipLaunchKernelGGL(link_decode_d128_kernel<false>, grid, dim3(64 * kWaves), 0, st, p);
  return hipGetLastError();
}

}  // namespace pic
