// Rows of a cache in pages (gfx950): where they lie, and the 8-bit format.
#pragma once
#include "common.hip.h"
#include "kernels.h"

namespace quoka {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The page of position `pos` of the sequence whose table row starts at `table`, for readers: some page of the pool whatever the entry.
__device__ __forceinline__ uint32_t page_of(const Pages& pg, const int32_t* table, int pos) {
  return min((uint32_t)table[min(pos >> pg.shift, pg.max_pages - 1)], (uint32_t)(pg.n_pages - 1));
}
__device__ __forceinline__ int slot_of(const Pages& pg, int pos) { return pos & ((1 << pg.shift) - 1); }
// Elements from the pool's start to a row, and the row's place among the scales (pools pass 2^32 bytes: 64 bits).
__device__ __forceinline__ long long row_at(const Pages& pg, uint32_t page, int kv, int slot) {
  return (long long)page * pg.st[0] + kv * pg.st[1] + slot * pg.st[2];
}
__device__ __forceinline__ long long scale_at(const Pages& pg, uint32_t page, int kv, int slot) {
  return (((long long)page * pg.n_kv + kv) << pg.shift) + slot;
}

// A row's power of two from its biased exponent, 1 .. 254.
__device__ __forceinline__ float row_scale(uint32_t e) { return __uint_as_float(e << 23); }
// The smallest power of two that brings magnitudes up to `top` to 448 = 1.75 * 2^8 or less, as a biased exponent: the exponent of `top`
// less 8, one more where its significand exceeds that of 448.  At least 1; at most 247, so 2^-e is a normal number too.
__device__ __forceinline__ uint32_t row_exponent(float top) {
  return (uint32_t)max((int)((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 8, 1);
}

// Eight 8-bit elements times a power of two.  To bfloat16 (four significant bits and a power of two: exact down to 2^-126), to float.
__device__ __forceinline__ u32x4 widen_bf16(u32x2 x, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], scale, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], scale, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], scale, true));
  return r;
}
__device__ __forceinline__ void widen_f32(uint32_t x, float scale, float* v) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  v[0] = lo[0] * scale;
  v[1] = lo[1] * scale;
  v[2] = hi[0] * scale;
  v[3] = hi[1] * scale;
}

}  // namespace quoka
