// A chunk's keys and values into the pages of a cache, and rows of the pages back out (the append step of Alg. 2 for a cache in
// pages; quoka_cache_write, quoka_cache_read).
//
// Bound by memory: every row is read once and written once.  A row is D / 8 lanes of eight elements, so the largest magnitude of a row,
// which sets the power of two of an 8-bit row, is found inside one row of 16 (D = 128) or 8 (D = 64) lanes with cross-lane moves, in
// registers; a thread has `U` rows on the way at once.  An 8-bit element is rounded once, to nearest even, by the conversion (the
// multiplication by a power of two before it is exact); widening is exact.
// Measured: 8 sequences of 2048 tokens, 8 heads of 128, bf16 to 8 bits 18.1 us (5.6 TB/s read and written), as they are 22.3 (6.0); 131072
// rows of 8 heads of 128 back from 8 bits 79 us (5.1 TB/s), 3 sequences up to 19999 of 4 heads of 64 as they are, K and V, 15.2 (5.9).  One
// token of 16 sequences 3 us, of which the launch and a chain of arguments, length, page and row are all.
#include "pages.hip.h"

namespace quoka {

constexpr int kPgThreads = 256;

// Largest value of the W lanes (8 or 16) that hold a row; every lane gets it.
template <int W>
__device__ __forceinline__ float row_max(float x) {
  uint32_t u = __float_as_uint(x);   // (magnitudes: their order is that of their bits)
  if constexpr (W == 16) return __uint_as_float(row16_max_u32(u));
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) u = max(u, (uint32_t)__shfl_xor((int)u, o, kWave));
  return __uint_as_float(u);
}

// Eight elements as a lane holds them, in memory's own form.
template <typename T>
struct Eight {
  u32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u32x4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e / 4][e % 4]);
    return __uint_as_float(e % 2 ? w[0][e / 2] & 0xFFFF0000u : w[0][e / 2] << 16);
  }
};

template <typename T, bool FP8, int D>
__device__ __forceinline__ void put_row(const Eight<T>& x, void* pages, uint8_t* scales, long long row, long long scale_row, bool on) {
  const int c = threadIdx.x % (D / 8);
  if constexpr (!FP8) {
    if (on) x.store(static_cast<T*>(pages) + row + 8 * c);
  } else {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x.at(e)));
    const uint32_t ex = row_exponent(row_max<D / 8>(top));
    const float by = row_scale(254u - ex);
    u32x2 q;
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x.at(0) * by, x.at(1) * by, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x.at(2) * by, x.at(3) * by, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x.at(4) * by, x.at(5) * by, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x.at(6) * by, x.at(7) * by, hi, true);
    q[0] = (uint32_t)lo;
    q[1] = (uint32_t)hi;
    if (on) {
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pages) + row + 8 * c) = q;
      if (c == 0) scales[scale_row] = (uint8_t)ex;
    }
  }
}

template <typename T, bool FP8, int D, int U>
__global__ __launch_bounds__(kPgThreads) void cache_write(Dims dm, Pages pg, const T* __restrict__ k, const T* __restrict__ v,
                                                          const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ chunk_lens) {
  constexpr int CG = D / 8, RPB = kPgThreads / CG;
  const int kv = (int)blockIdx.y % dm.n_kv, b = (int)blockIdx.y / dm.n_kv;
  const int r0 = threadIdx.x / CG, c = threadIdx.x % CG;
  const int C = chunk_lens == nullptr ? dm.C : min(chunk_lens[b], dm.C);
  const int first = (int)blockIdx.x * RPB * U;
  if (first >= C) return;   // block-uniform
  const T* kc = k + b * dm.cks[0] + kv * dm.cks[1] + 8 * c;
  const T* vc = v + b * dm.cks[0] + kv * dm.cks[1] + 8 * c;
  Eight<T> xk[U], xv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long at = (long long)min(first + u * RPB + r0, C - 1) * dm.cks[2];
    xk[u].load(kc + at);
    xv[u].load(vc + at);
  }
  const int pos0 = min(max(kv_lens[b], 0), dm.T_max);
  const int32_t* table = pg.table + (long long)b * pg.max_pages;
  uint32_t page[U];
#pragma unroll
  for (int u = 0; u < U; ++u) page[u] = (uint32_t)table[min((pos0 + min(first + u * RPB + r0, C - 1)) >> pg.shift, pg.max_pages - 1)];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = first + u * RPB + r0, pos = pos0 + i;
    const bool on = i < C && page[u] < (uint32_t)pg.n_pages && (pos >> pg.shift) < pg.max_pages;
    const long long row = row_at(pg, page[u], kv, slot_of(pg, pos)), srow = scale_at(pg, page[u], kv, slot_of(pg, pos));
    put_row<T, FP8, D>(xk[u], pg.k, pg.k_scale, row, srow, on);
    put_row<T, FP8, D>(xv[u], pg.v, pg.v_scale, row, srow, on);
  }
}

// blockIdx.z: K or V (the first that is wanted, then the other).
template <typename T, bool FP8, int D, int U>
__global__ __launch_bounds__(kPgThreads) void cache_read(Dims dm, Pages pg, const int32_t* __restrict__ kv_lens, T* __restrict__ k,
                                                         T* __restrict__ v) {
  constexpr int CG = D / 8, RPB = kPgThreads / CG;
  const int kv = (int)blockIdx.y % dm.n_kv, b = (int)blockIdx.y / dm.n_kv;
  const int r0 = threadIdx.x / CG, c = threadIdx.x % CG;
  const bool is_v = k == nullptr || blockIdx.z == 1;
  const int T_b = min(max(kv_lens[b], 0), dm.T_max);
  const int first = (int)blockIdx.x * RPB * U;
  if (first >= T_b) return;   // block-uniform
  const int32_t* table = pg.table + (long long)b * pg.max_pages;
  const void* pages = is_v ? pg.v : pg.k;
  const uint8_t* scales = is_v ? pg.v_scale : pg.k_scale;
  T* out = (is_v ? v : k) + b * dm.kvs[0] + kv * dm.kvs[1] + 8 * c;
  uint32_t page[U];
#pragma unroll
  for (int u = 0; u < U; ++u) page[u] = page_of(pg, table, min(first + u * RPB + r0, T_b - 1));
  if constexpr (!FP8) {
    Eight<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u].load(static_cast<const T*>(pages) + row_at(pg, page[u], kv, slot_of(pg, min(first + u * RPB + r0, T_b - 1))) + 8 * c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = first + u * RPB + r0;
      if (t < T_b) x[u].store(out + t * dm.kvs[2]);
    }
  } else {
    u32x2 x[U];
    uint32_t e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int slot = slot_of(pg, min(first + u * RPB + r0, T_b - 1));
      x[u] = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pages) + row_at(pg, page[u], kv, slot) + 8 * c);
      e[u] = scales[scale_at(pg, page[u], kv, slot)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = first + u * RPB + r0;
      Eight<T> y;
      if constexpr (sizeof(T) == 2) {
        y.w[0] = widen_bf16(x[u], row_scale(e[u]));
      } else {
        float f[8];
        widen_f32(x[u][0], row_scale(e[u]), f);
        widen_f32(x[u][1], row_scale(e[u]), f + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) y.w[i / 4][i % 4] = __float_as_uint(f[i]);
      }
      if (t < T_b) y.store(out + t * dm.kvs[2]);
    }
  }
}

template <typename T, bool FP8, int D>
static hipError_t launch_write_d(const Dims& dm, const Pages& pg, const void* k, const void* v, const int32_t* kv_lens,
                                 const int32_t* chunk_lens, hipStream_t st) {
  // (1, 2, 4: the first two launches above 18.2, 18.1, 17.7 and 22.5, 22.3, 20.9 us; one token of 16 sequences 3.0 with 2 and 3.4 with 4, 3
  // sequences of 57 - 333 float32 rows of 3 heads of 64 as they are 3.4 and 4.1)
  constexpr int U = 2, ROWS = kPgThreads / (D / 8) * U;
  hipLaunchKernelGGL((cache_write<T, FP8, D, U>), dim3((dm.C + ROWS - 1) / ROWS, dm.b * dm.n_kv), dim3(kPgThreads), 0, st, dm, pg,
                     static_cast<const T*>(k), static_cast<const T*>(v), kv_lens, chunk_lens);
  return hipGetLastError();
}

template <typename T, bool FP8, int D>
static hipError_t launch_read_d(const Dims& dm, const Pages& pg, const int32_t* kv_lens, void* k, void* v, hipStream_t st) {
  constexpr int U = 4, ROWS = kPgThreads / (D / 8) * U;   // (2, 4, 8: 87.2, 79.8, 80.5 us and 15.2, 15.4, 16.0)
  hipLaunchKernelGGL((cache_read<T, FP8, D, U>), dim3((dm.T_max + ROWS - 1) / ROWS, dm.b * dm.n_kv, k != nullptr && v != nullptr ? 2 : 1),
                     dim3(kPgThreads), 0, st, dm, pg, kv_lens, static_cast<T*>(k), static_cast<T*>(v));
  return hipGetLastError();
}

hipError_t launch_cache_write(const Dims& dm, int dtype, bool fp8, const Pages& pg, const void* k, const void* v, const int32_t* kv_lens,
                              const int32_t* chunk_lens, hipStream_t st) {
  auto launch = [&](auto one) {
    using T = decltype(one);
    if (dm.d == 64)
      return fp8 ? launch_write_d<T, true, 64>(dm, pg, k, v, kv_lens, chunk_lens, st)
                 : launch_write_d<T, false, 64>(dm, pg, k, v, kv_lens, chunk_lens, st);
    return fp8 ? launch_write_d<T, true, 128>(dm, pg, k, v, kv_lens, chunk_lens, st)
               : launch_write_d<T, false, 128>(dm, pg, k, v, kv_lens, chunk_lens, st);
  };
  return dtype == QUOKA_BF16 ? launch(uint16_t{}) : launch(float{});
}

hipError_t launch_cache_read(const Dims& dm, int dtype, bool fp8, const Pages& pg, const int32_t* kv_lens, void* k, void* v,
                             hipStream_t st) {
  auto launch = [&](auto one) {
    using T = decltype(one);
    if (dm.d == 64) return fp8 ? launch_read_d<T, true, 64>(dm, pg, kv_lens, k, v, st) : launch_read_d<T, false, 64>(dm, pg, kv_lens, k, v, st);
    return fp8 ? launch_read_d<T, true, 128>(dm, pg, kv_lens, k, v, st) : launch_read_d<T, false, 128>(dm, pg, kv_lens, k, v, st);
  };
  return dtype == QUOKA_BF16 ? launch(uint16_t{}) : launch(float{});
}

}  // namespace quoka
