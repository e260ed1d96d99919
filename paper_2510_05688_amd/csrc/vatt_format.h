// Formats of the KV cache's rows: where a row and its scales lie, and the conversions.
//
//   bf16   2 d bytes per row
//   e4m3   d bytes per row:   sign, 4 exponent bits (bias 7), 3 of the mantissa; largest 448
//   e2m1   d / 2 bytes per row: sign, 2 exponent bits (bias 1), 1 of the mantissa; 0 .5 1 1.5 2 3 4 6; column 2 j in the lower
//          half of byte j
// The last two have one scale byte per 32 columns, the power of two 2^(byte - 127); 255 makes the group NaN.  The codes of all rows
// come first, in the order of the bf16 layout, then the scale bytes of all rows (d / 32 each), which in the contiguous layout leave
// room for a multiple of 8 rows per KV head, so that the scales of four rows are one aligned load.
// Every code times its scale is a bf16 number (4 significant bits), so what a cache holds goes into the bf16 matrix instructions as it is.
#pragma once

#include "vatt_dev.h"
#include "vatt_internal.h"

namespace vatt {

template <int FMT, int D>
constexpr int kRowBytes = FMT == VATT_KV_BF16 ? 2 * D : FMT == VATT_KV_E4M3 ? D : D / 2;

// Physical rows of a cache.
struct RowMap {
  const int32_t* block_table;
  int32_t n_max, n_scales;  // contiguous: rows, and rows of scales, per KV head
  int32_t Hkv, page_shift, pages_per_seq, num_blocks;
};

struct RowAt {
  int64_t row, scales;
};

template <bool PAGED>
__device__ __forceinline__ int row_block(const RowMap& M, int b, int tok) {
  if constexpr (PAGED) return min(max(M.block_table[(int64_t)b * M.pages_per_seq + (tok >> M.page_shift)], 0), M.num_blocks - 1);
  else return 0;
}
template <bool PAGED>
__device__ __forceinline__ RowAt row_at(const RowMap& M, int b, int kvh, int tok, int blk) {
  if constexpr (PAGED) {
    const int64_t r = (((int64_t)blk * M.Hkv + kvh) << M.page_shift) + (tok & ((1 << M.page_shift) - 1));
    return {r, r};
  } else {
    const int64_t head = (int64_t)b * M.Hkv + kvh;
    return {head * M.n_max + tok, head * M.n_scales + tok};
  }
}

inline RowMap row_map(const Plan& pl, const int32_t* block_table) {
  RowMap M;
  M.block_table = block_table;
  M.n_max = pl.p.n_max;
  M.n_scales = (pl.p.n_max + 7) / 8 * 8;
  M.Hkv = pl.p.n_kv_heads;
  M.page_shift = pl.kv_k.page_shift;
  M.pages_per_seq = pl.kv_k.pages_per_seq;
  M.num_blocks = pl.p.num_blocks;
  return M;
}

typedef __bf16 bf16x2_f __attribute__((ext_vector_type(2)));
typedef short i16x2_f __attribute__((ext_vector_type(2)));

// Two fp32 values rounded to bf16 (nearest, ties to even), the first in the lower half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2_f r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }  // (0 is read as 2^-127 by the conversions)

// Codes of a 32-bit word to bf16 pairs: four e4m3 values, or pair `I` of eight e2m1 values.  Exact; NaN with scale byte 255.
__device__ __forceinline__ uint2 e4m3_to_bf16(uint32_t codes, float scale) {
  const bf16x2_f lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  const bf16x2_f hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
template <int I>
__device__ __forceinline__ uint32_t e2m1_to_bf16(uint32_t codes, float scale) {
  const bf16x2_f r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, I);
  return __builtin_bit_cast(uint32_t, r);
}

// The 8 consecutive columns of a row that one lane has, as codes.
template <int FMT>
struct Chunk {
  uint32_t w[FMT == VATT_KV_BF16 ? 4 : FMT == VATT_KV_E4M3 ? 2 : 1];
};
template <int FMT>
__device__ __forceinline__ Chunk<FMT> load_chunk(const unsigned char* p) {
  Chunk<FMT> c;
  if constexpr (FMT == VATT_KV_BF16) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    c.w[0] = x.x; c.w[1] = x.y; c.w[2] = x.z; c.w[3] = x.w;
  } else if constexpr (FMT == VATT_KV_E4M3) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    c.w[0] = x.x; c.w[1] = x.y;
  } else {
    c.w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  return c;
}
template <int FMT>
__device__ __forceinline__ void store_chunk(unsigned char* p, const Chunk<FMT>& c) {
  if constexpr (FMT == VATT_KV_BF16) *reinterpret_cast<uint4*>(p) = make_uint4(c.w[0], c.w[1], c.w[2], c.w[3]);
  else if constexpr (FMT == VATT_KV_E4M3) *reinterpret_cast<uint2*>(p) = make_uint2(c.w[0], c.w[1]);
  else *reinterpret_cast<uint32_t*>(p) = c.w[0];
}
template <int FMT>
__device__ __forceinline__ uint4 chunk_bf16(const Chunk<FMT>& c, uint32_t scale_byte) {
  if constexpr (FMT == VATT_KV_BF16) {
    return make_uint4(c.w[0], c.w[1], c.w[2], c.w[3]);
  } else if constexpr (FMT == VATT_KV_E4M3) {
    const float s = scale_of(scale_byte);
    const uint2 a = e4m3_to_bf16(c.w[0], s), b = e4m3_to_bf16(c.w[1], s);
    return make_uint4(a.x, a.y, b.x, b.y);
  } else {
    const float s = scale_of(scale_byte);
    return make_uint4(e2m1_to_bf16<0>(c.w[0], s), e2m1_to_bf16<1>(c.w[0], s), e2m1_to_bf16<2>(c.w[0], s), e2m1_to_bf16<3>(c.w[0], s));
  }
}

// Quantises 8 columns, together with the three other lanes of the quad that hold the rest of their 32.  The scale is the smallest
// power of two at which no magnitude is above the format's largest value, so that nothing is cut off; rounding is to the nearest, ties to
// even: half a step of the format (e4m3 2^-4 of a value, e2m1 2^-2), which is what a cache in 8 or 4 bits costs.  Magnitudes are limited
// to 1.5 * 2^127 first (above it a rounded value could leave bf16).  A group with an Inf or a NaN gets scale byte 255.
template <int FMT>
__device__ __forceinline__ Chunk<FMT> quantise(const float (&y)[8], uint32_t& scale_byte) {
  static_assert(FMT != VATT_KV_BF16, "a quantised format");
  constexpr float kLargest = 1.5f * 1.7014118346046923e38f;
  uint32_t top = 0;  // (magnitudes as integers are in the order of the numbers, Inf and NaN on top)
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
  top = max(top, dpp_u32<0xB1>(top));
  top = max(top, dpp_u32<0x4E>(top));
  const bool finite = top < 0x7f800000u;
  top = min(top, __float_as_uint(kLargest));
  const int x = (int)(top >> 23);
  const uint32_t mant = top & 0x7fffffu;
  const int e = FMT == VATT_KV_E4M3 ? x - 8 + (mant > 0x600000u ? 1 : 0)   // 448 = 1.75 * 2^8
                                    : x - 2 + (mant > 0x400000u ? 1 : 0);  // 6 = 1.5 * 2^2
  const uint32_t byte = (uint32_t)max(e, 0);
  scale_byte = finite ? byte : 255u;
  const float s = scale_of(byte);
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = finite ? fminf(fmaxf(y[i], -kLargest), kLargest) : 0.f;
  Chunk<FMT> c;
  if constexpr (FMT == VATT_KV_E4M3) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i16x2_f r = {0, 0};
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, z[4 * h], z[4 * h + 1], s, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, z[4 * h + 2], z[4 * h + 3], s, true);
      c.w[h] = __builtin_bit_cast(uint32_t, r);
    }
  } else {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, z[0], z[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, z[2], z[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, z[4], z[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, z[6], z[7], s, 3);
    c.w[0] = r;
  }
  return c;
}

}  // namespace vatt
