// The 4-bit chunk cache: number format, tile layout, and the conversions its
// kernels share.
//
// Format. A row (one token of one head, K or V) is cut into blocks of 32
// elements. A block holds e2m1 numbers (sign and 0, 0.5, 1, 1.5, 2, 3, 4, 6)
// times one power of two 2^e, kept as the byte e + 127. With a = max |x| of the
// block, e is the smallest exponent with a < 7 * 2^e: the largest element then
// rounds to at most 6 * 2^e, by no more than half a step of a grid without an
// end (a rule that takes e from the exponent of a alone cuts elements between 7
// and 8 times 2^e off by up to a quarter). e is held to -126 .. 125, so
// that 2^e is a normal fp32 number and 6 * 2^e a finite bf16 one: smaller
// blocks lose bits, and infinities become the largest number. Elements are
// rounded to nearest, ties to even. A block that holds a NaN gets the byte
// 255 and reads as NaN throughout. Every other value is a bf16 number, so
// that widening a block to bf16 is exact. 17 bytes hold 32 elements.
//
// Blocks lie along a row, for V too, though its product runs along the tokens:
// a row's bytes then depend on nothing but the row, and rows can be written one
// by one (pic_store_write_rows).
#pragma once

#include "pic_internal.hpp"

namespace pic {

// Tile layout, 64 tokens of one head, D elements wide: the codes in the order
// in which lane l = 16 g + m of a wave takes them as operands of
// v_mfma_f32_16x16x32_bf16, 16 bytes (a unit) per load and lane, so that every
// load of a wave is 1 KB in one piece.
//   K codes  D * 32 bytes. For the product K . Q^T lane (m, g) feeds D/4
//            elements from D/4 * g on of the keys 16 b + m, b = 0..3 (the order of
//            the D steps of a sum is free, q follows it): D/8 bytes per key,
//            one key (D = 128) or two, b and b + 1 (D = 64), per unit.
//   V codes  D * 32 bytes. For V^T . P^T lane (m, g) feeds D/16 channels from
//            D/16 * m on of the keys 16 b + 4 g + i, i = 0..3, which are the keys whose
//            scores it holds after the first product: D/32 bytes per key, four
//            keys (D = 128) or eight per unit.
//   K scales 64 * D/32 bytes, [block c][m][b]
//   V scales 64 * D/32 bytes, [g][block c][b][i]
// Tiles of a page follow each other head by head: [page][head][tile].
template <int D>
struct Fp4Tile {
  static_assert(D == 64 || D == 128, "head widths of the 4-bit kernels");
  static constexpr int kBlocks = D / 32;                 // blocks of a row
  static constexpr int kCode = D * 32;                   // bytes of K (or V) codes
  static constexpr int kV = kCode, kKs = 2 * kCode, kVs = kKs + 64 * kBlocks;
  static constexpr int kBytes = kVs + 64 * kBlocks;
  static_assert(kBytes == 68 * D, "17 bytes per 32 elements");
  // Byte that holds elements e and e + 1 (e even) of a key, and the scale
  // byte of its block c.
  __host__ __device__ static constexpr int k_code(int key, int e) {
    return D == 128 ? ((key >> 4) * 64 + (e >> 5) * 16 + (key & 15)) * 16 + (e & 31) / 2
                    : ((key >> 5) * 64 + (e >> 4) * 16 + (key & 15)) * 16 + ((key >> 4) & 1) * 8 +
                          (e & 15) / 2;
  }
  __host__ __device__ static constexpr int v_code(int key, int e) {
    return D == 128
               ? kV + ((key >> 4) * 64 + ((key >> 2) & 3) * 16 + (e >> 3)) * 16 + (key & 3) * 4 +
                     (e & 7) / 2
               : kV + ((key >> 5) * 64 + ((key >> 2) & 3) * 16 + (e >> 2)) * 16 +
                     (((key >> 4) & 1) * 4 + (key & 3)) * 2 + (e & 3) / 2;
  }
  __host__ __device__ static constexpr int k_scale(int key, int c) {
    return kKs + (c * 16 + (key & 15)) * 4 + (key >> 4);
  }
  __host__ __device__ static constexpr int v_scale(int key, int c) {
    return kVs + (((key >> 2) & 3) * kBlocks + c) * 16 + (key >> 4) * 4 + (key & 3);
  }
};

// Head widths of a 4-bit store.
inline bool fp4_width(int d_k, int d_v) { return d_k == d_v && (d_k == 64 || d_k == 128); }
// Bytes of one page: 64 tokens of every head.
inline int64_t fp4_page_bytes(int64_t heads, int64_t d) { return heads * 68 * d; }

// A call's tables in its kernel's arguments, read where they are: no kernel copies them
// first.
struct Fp4Args {
  LinkParams p;
  Fp4Tabs t;
};
// What a workgroup starts a pass over its piece from: its kernel's arguments (LinkParams first),
// its number, and this thread's lane and wave. kArg: the tables follow in the arguments. All but
// the wave are read anew for every pass, so that nothing formed from them is kept for the
// next one.
template <bool kArg>
struct Fp4Start {
  typedef __attribute__((address_space(4))) const char *const_bytes;
  LinkParams p;
  const WorkItem *items;
  const_links links;
  int block, lane, wave;
  __device__ __forceinline__ explicit Fp4Start(int wave_) : wave(wave_) {
    const_bytes args = (const_bytes)__builtin_amdgcn_kernarg_segment_ptr();
    block = blockIdx.x;
    int all = -1;
    asm volatile("" : "+s"(args), "+s"(block), "+s"(all));
    lane = __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0));
#ifdef __HIP_DEVICE_COMPILE__    // (no copies between address spaces on the host)
    p = *(__attribute__((address_space(4))) const LinkParams *)args;
#endif
    if (kArg) {
      const const_bytes t = args + offsetof(Fp4Args, t);
      items = (const WorkItem *)t;
      links = (const_links)(t + p.n_items * (int)sizeof(WorkItem));
    } else {
      items = p.items;
      links = (const_links)p.links;
    }
  }
};

// Walk over the links of a work item. kAhead: the next link's entry is read when
// the one before begins, so that no tile waits for a table (narrow_heads 143 -> 136
// us); the 128-wide 256-row kernel, bound by its products, loses 1% by it.
// (lp of a 4-bit item: links that follow the first.)
template <bool kAhead>
struct LinkCursor {
  const_links at;          // the current link
  int left;                // links after it
  const char *base;        // its first tile
  int len, tok0, tile0, end;
  const char *next_base;
  int next_len, next_tok0, next_tile0;

  __device__ __forceinline__ void read(const_links n) {
    next_base = (const char *)n->k;
    next_len = n->len;
    next_tok0 = n->tok0;
    next_tile0 = n->tile0;
  }
  __device__ __forceinline__ void start(const_links links, const WorkItem &it) {
    at = links + it.link;
    left = it.lp;
    base = (const char *)it.k;
    len = it.len;
    tok0 = it.tok0;
    tile0 = it.tile0;
    end = tile0 + (len + kTile - 1) / kTile;
    // (an empty piece names no link to walk from)
    if (kAhead && it.t_begin < it.t_end) read(at + (left > 0 ? 1 : 0));
  }
  __device__ __forceinline__ void next() {
    ++at;
    if (!kAhead) read(at);
    base = next_base;
    len = next_len;
    tok0 = next_tok0;
    tile0 = next_tile0;
    end = tile0 + (len + kTile - 1) / kTile;
    if (kAhead) read(at + (--left > 0 ? 1 : 0));
  }
};

// Large values. A sum of values times probabilities at most 1 leaves the fp32 range where two
// of 6 * 2^125 meet, though their mean does not, and sooner where the maximum lags behind. A
// workgroup whose sums come out too large or NaN takes its piece again, against the exact
// maximum plus fp4_bias: each of the piece's n < 2^bias probabilities is then at most 2^-bias,
// and no sum exceeds the largest value. What that loses are probabilities below 2^(bias - 126),
// as the first pass loses those below 2^-126. Outputs, log-sum-exp and the merge of pieces see
// one power of two in maximum and sums, and need nothing more. Both passes are the same code (a
// second copy of it made the compiler spill 82 registers); the check costs an instruction per
// two sums at the end of a piece.
__device__ __forceinline__ float fp4_bias(int tiles) {
  return (float)(32 - __builtin_clz(tiles * kTile));
}

typedef __bf16 fp4_bf16x2 __attribute__((ext_vector_type(2)));

// The scale byte of a block from the largest |x| of its bf16 patterns (sign
// cleared; NaN patterns compare above infinity's).
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax) {
  const int e = (int)(amax >> 7) - 2 + ((amax & 127) >= 96 ? 1 : 0);   // 1.75 and above: one more
  return amax > 0x7f80u ? 255u : (uint32_t)(e < 1 ? 1 : e > 252 ? 252 : e);
}
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// 8 bf16 numbers to 8 codes (the conversion divides by the scale, rounds to
// nearest even and ends at 6).
__device__ __forceinline__ uint32_t fp4_encode8(uint4 x, float scale) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.x), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.y), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.z), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(fp4_bf16x2, x.w), scale, 3);
}
// Codes 2 kSel and 2 kSel + 1 of c as a pair of bf16 numbers (one instruction,
// exact; NaN where the scale is not finite).
template <int kSel>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t c, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, kSel));
}
__device__ __forceinline__ uint4 fp4_decode8(uint32_t c, float scale) {
  return make_uint4(fp4_pair<0>(c, scale), fp4_pair<1>(c, scale), fp4_pair<2>(c, scale),
                    fp4_pair<3>(c, scale));
}

}  // namespace pic
