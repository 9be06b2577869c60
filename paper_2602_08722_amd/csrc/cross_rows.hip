// Cross attention of a few query rows (at most four per KV head) over states in pages: a block has a sequence and a KV head to
// itself and writes the rows whole.
//
// Sixteen lanes have a state: lane c elements 4 c .. + 3 of every 64, of K, V, the query rows and their sums, so that loads are whole rows,
// a logit is a sum over a row of 16 lanes, and every group of lanes has an online softmax of its own over its states; the groups' sums meet
// at the end.  (The 32-row blocks of the matrix instructions would be mostly padding.)  A wave has four groups and takes tiles of 4 U
// neighbouring states in turn with the block's others.
// Bound by a chain of fetches (length, pages, rows: 4 us), then, one row and one sequence, by the vector unit (4.5 us for 1000 states at d 64,
// 9 at d 128; four rows 11 and 17), and batches by memory.  Measured, float32, one token: 8 sequences of 300 states, 12 heads, d 64 5.2 us
// (attn_f32 13.1), of 1000 11.5 (22.7), 32 of 4000 144 (192; 5.4 TB/s); 32 of 1000, 8 heads of 4, d 128 43 (55).  Sixteen waves of half as many states
// on the way: 0.3 - 0.9 us longer for short lists, the same for long ones; sixteen of as many 0.7 - 3 longer.
#include <atomic>
#include <type_traits>

#include "pages.hip.h"

namespace quoka {

__device__ __forceinline__ void store_four(float* at, float4 x) { *reinterpret_cast<float4*>(at) = x; }
__device__ __forceinline__ void store_four(uint16_t* at, float4 x) {
  const bf16x2 lo = {(__bf16)x.x, (__bf16)x.y}, hi = {(__bf16)x.z, (__bf16)x.w};   // (the output's one rounding; probabilities have none here)
  *reinterpret_cast<u32x2*>(at) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// Four elements as a row keeps them: in 8 bits with their row's exponent, in bfloat16, in float32.
__device__ __forceinline__ void widen(uint32_t x, uint32_t exponent, float* y) { widen_f32(x, row_scale(exponent), y); }
typedef uint32_t u32x1 __attribute__((ext_vector_type(1)));
__device__ __forceinline__ void widen(u32x1 x, uint32_t exponent, float* y) { widen_f32(x[0], row_scale(exponent), y); }
__device__ __forceinline__ void widen(u32x2 x, uint32_t, float* y) {
  y[0] = __uint_as_float(x[0] << 16), y[1] = __uint_as_float(x[0] & 0xFFFF0000u);
  y[2] = __uint_as_float(x[1] << 16), y[3] = __uint_as_float(x[1] & 0xFFFF0000u);
}
__device__ __forceinline__ void widen(u32x4 x, uint32_t, float* y) {
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = __uint_as_float(x[e]);
}

template <typename T>
using four_of = std::conditional_t<sizeof(T) == 4, u32x4, u32x2>;

// T: of queries, outputs and rows that are not in 8 bits.
template <typename T, int D, bool FP8, int R, int WAVES, int U>
__global__ __launch_bounds__(64 * WAVES) void cross_rows(Dims dm, PagedArgs a) {
  constexpr int LPR = 16, G = kWave / LPR, NQ = D / 64, TILE = G * U, THREADS = 64 * WAVES;   // NQ: fours of elements of a lane
  static_assert(U <= 8, "row16_lane");
  extern __shared__ __align__(16) unsigned char smem[];
  float* mo = reinterpret_cast<float*>(smem);   // [WAVES][R][D]
  float* mm = mo + WAVES * R * D;               // [WAVES][R]
  float* ml = mm + WAVES * R;
  float* mw = ml + WAVES * R;
  const Pages& pg = a.pg;
  const int b = blockIdx.x, kv = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane % LPR, group = lane / LPR;
  const int g = dm.g;
  const int C = a.chunk_lens == nullptr ? dm.C : max(min(a.chunk_lens[b], dm.C), 0);
  const int n = min(max(a.kv_lens[b], 0), dm.T_max), n_rows = n > 0 ? C * g : 0;   // n_rows <= R, checked by the launcher
  // rows past the chunk, and all where there is nothing to see: zeros and no weight
  for (int i = n_rows * (D / 4) + tid; i < dm.C * g * (D / 4); i += THREADS) {
    const int r = i / (D / 4), c4 = i % (D / 4), tok = r / g, h = kv * g + r % g;
    store_four(static_cast<T*>(a.out) + b * dm.os[0] + h * dm.os[1] + (size_t)tok * dm.os[2] + 4 * c4, make_float4(0.f, 0.f, 0.f, 0.f));
    if (c4 == 0 && a.lse != nullptr) a.lse[(size_t)(b * dm.n_q + h) * dm.C + tok] = -INFINITY;
  }
  if (n_rows == 0) return;   // block-uniform

  const int32_t* table = pg.table + (size_t)b * pg.max_pages;
  constexpr int es = FP8 ? 1 : (int)sizeof(T);
  const char* k_pool = static_cast<const char*>(pg.k) + (size_t)kv * pg.st[1] * es;
  const char* v_pool = static_cast<const char*>(pg.v) + (size_t)kv * pg.st[1] * es;
  const uint8_t* k_scales = FP8 ? pg.k_scale + ((size_t)kv << pg.shift) : nullptr;
  const uint8_t* v_scales = FP8 ? pg.v_scale + ((size_t)kv << pg.shift) : nullptr;
  const uint32_t page_units = (uint32_t)(pg.st[0] / (16 / es)), slot_units = (uint32_t)(pg.st[2] / (16 / es)), page_scales = (uint32_t)pg.n_kv << pg.shift;
  // Lane c < U of a group looks up its state c of a tile; lane groups take neighbouring ones.  (Past the end: the last state, masked below.)
  uint32_t pos = 0, page = 0;
  auto look_up = [&](int t0) __attribute__((always_inline)) {
    pos = (uint32_t)min(t0 + (c % U) * G + group, n - 1);
    page = (uint32_t)table[min((int)(pos >> pg.shift), pg.max_pages - 1)];
  };
  int t0 = w * TILE;
  look_up(t0);

  float q[R][NQ][4], o[R][NQ][4], m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = r < n_rows ? r : 0;   // (padding rows repeat the first and are never stored)
    const T* at = static_cast<const T*>(a.q) + b * dm.qs[0] + (size_t)(kv * g + row % g) * dm.qs[1] + (size_t)(row / g) * dm.qs[2] + 4 * c;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      widen(*reinterpret_cast<const four_of<T>*>(at + 64 * j), 0u, q[r][j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[r][j][e] = 0.f;
    }
    m[r] = -INFINITY;
    l[r] = 0.f;
  }
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);   // the softmax scale and the change to base 2
  for (; t0 < n; t0 += WAVES * TILE) {
    const uint32_t at_page = min(page, (uint32_t)(pg.n_pages - 1)), slot = pos & ((1u << pg.shift) - 1u);
    const uint32_t off = at_page * page_units + slot * slot_units;
    float kx[U][NQ][4], vx[U][NQ][4];
    uint32_t ex = 0;
    if constexpr (FP8) {
      const uint32_t s = at_page * page_scales + slot;
      ex = (uint32_t)k_scales[s] | (uint32_t)v_scales[s] << 8;
    }
    typedef uint32_t held __attribute__((ext_vector_type(es)));   // four elements as they are kept
    held kr[U][NQ], vr[U][NQ];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = (size_t)row16_lane(off, u) * 16 + (size_t)(4 * es) * c;
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        kr[u][j] = *reinterpret_cast<const held*>(k_pool + at + 64 * es * j);
        vr[u][j] = *reinterpret_cast<const held*>(v_pool + at + 64 * es * j);
      }
    }
    const int left = n - t0 - group;   // state u of the group is there if u * G < left
    if (t0 + WAVES * TILE < n) look_up(t0 + WAVES * TILE);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t e = FP8 ? row16_lane(ex, u) : 0u;
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        widen(kr[u][j], e & 255u, kx[u][j]);
        widen(vr[u][j], e >> 8, vx[u][j]);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s[U], top = m[r];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) dot = fmaf(q[r][j][e], kx[u][j][e], dot);
        s[u] = u * G < left ? row16_sum(dot) * sl2 : -INFINITY;
        top = fmaxf(top, s[u]);
      }
      const float ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m[r] - ref);
      m[r] = top;
      l[r] *= alpha;
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[r][j][e] *= alpha;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float p = __builtin_amdgcn_exp2f(s[u] - ref);
        l[r] += p;
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][j][e] = fmaf(p, vx[u][j][e], o[r][j][e]);
      }
    }
  }

  // ---- the groups of a wave, then the waves ----
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float top = fmaxf(m[r], __shfl_xor(m[r], 16, kWave));
    top = fmaxf(top, other_half(top));
    const float wgt = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r] - top);
    l[r] *= wgt;
    l[r] += __shfl_xor(l[r], 16, kWave);
    l[r] += other_half(l[r]);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = o[r][j][e] * wgt;
        x += __shfl_xor(x, 16, kWave);
        o[r][j][e] = x + other_half(x);
      }
      if (group == 0) *reinterpret_cast<float4*>(mo + (w * R + r) * D + 64 * j + 4 * c) = make_float4(o[r][j][0], o[r][j][1], o[r][j][2], o[r][j][3]);
    }
    if (lane == 0) {
      mm[w * R + r] = top;
      ml[w * R + r] = l[r];
    }
  }
  __syncthreads();
  if (tid < n_rows) {   // the weights of a row's waves, divided by its sum (the first wave has seen a state: finite)
    float top = mm[tid], sum = 0.f, e[WAVES];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = fmaxf(top, mm[i * R + tid]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      e[i] = mm[i * R + tid] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mm[i * R + tid] - top);
      sum += e[i] * ml[i * R + tid];
    }
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mw[i * R + tid] = e[i] / sum;
    if (a.lse != nullptr) a.lse[(size_t)(b * dm.n_q + kv * g + tid % g) * dm.C + tid / g] = (top + log2f(sum)) * 0.6931471805599453f;
  }
  __syncthreads();
  for (int i = tid; i < n_rows * (D / 4); i += THREADS) {
    const int r = i / (D / 4), c4 = i % (D / 4);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const float wgt = mw[k * R + r];
      const float4 x = *reinterpret_cast<const float4*>(mo + (k * R + r) * D + 4 * c4);
      acc.x += wgt * x.x;
      acc.y += wgt * x.y;
      acc.z += wgt * x.z;
      acc.w += wgt * x.w;
    }
    store_four(static_cast<T*>(a.out) + b * dm.os[0] + (kv * g + r % g) * dm.os[1] + (size_t)(r / g) * dm.os[2] + 4 * c4, acc);
  }
}

// bfloat16: where rows are one or two and states few, or sequences many, less than the kernels of matrix instructions (cross_few, paged_decode).
// Us of this one and those: one row, 8 sequences, 12 heads, d 64, 40 states 4.2 / 5.4, 300 5.2 / 6.4, 600 6.6 / 7.2, 1000 9.1 / 8.8, d 128, 300 6.1 / 7.0,
// 600 9.2 / 9.3; 100 sequences of 100, d 64 8.3 / 16.0, 1000 46.6 / 54.5, 2000 85 / 95; two rows, 8 sequences, 8 heads, d 64, 100 5.1 / 5.4, 300 6.3 / 6.4,
// d 128, 40 5.0 / 5.5, 100 5.9 / 5.9; 100 of 100, d 64 10.3 / 14.0, 600 24.9 / 27.2, 1000 37.1 / 38.5; four rows 1.1 - 2 of the time nearly everywhere.
bool cross_rows_take_bf16(const Dims& dm) {
  const long long rows = (long long)dm.C * dm.g;
  const bool many = (long long)dm.b * dm.n_kv > 256, wide = dm.d == 128;
  if (rows > 2) return false;
  return dm.T_max <= (rows <= 1 ? many ? 1000 : wide ? 400 : 600 : many ? 600 : wide ? 50 : 150);
}

// Us of a call in float32, roughly: by the states that a row sees and by rounds of blocks (infinity: not for this kernel).
float cross_rows_us(const Dims& dm) {
  const long long rows = (long long)dm.C * dm.g, rounds = ((long long)dm.b * dm.n_kv + 255) / 256;   // (compute units)
  if (rows > 4) return INFINITY;
  constexpr float kFixed[2][3] = {{4.0f, 4.5f, 5.5f}, {4.0f, 4.4f, 5.6f}}, kState[2][3] = {{0.0045f, 0.006f, 0.011f}, {0.0095f, 0.0095f, 0.0165f}};
  const int wide = dm.d == 128 ? 1 : 0, at = rows <= 1 ? 0 : rows <= 2 ? 1 : 2;
  return (float)rounds * (kFixed[wide][at] + kState[wide][at] * (float)dm.T_max);
}

hipError_t launch_cross_rows(const Dims& dm, int dtype, bool fp8, const PagedArgs& a, hipStream_t st) {
  auto launch = [&](auto type, auto d, auto eight_bit, auto rows) -> hipError_t {
    using T = decltype(type);
    constexpr int D = decltype(d)::value, R = decltype(rows)::value, WAVES = 8, U = D == 64 ? 8 : 4;
    constexpr bool FP8 = decltype(eight_bit)::value;
    constexpr size_t lds = (size_t)WAVES * R * (D + 3) * 4;
    static std::atomic<uint64_t> lds_done{0};
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&cross_rows<T, D, FP8, R, WAVES, U>), lds, lds_done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_rows<T, D, FP8, R, WAVES, U>), dim3(dm.b, dm.n_kv), dim3(64 * WAVES), lds, st, dm, a);
    return hipGetLastError();
  };
  using std::integral_constant;
  const int n = dm.C * dm.g;
  auto with_rows = [&](auto type, auto d, auto eight_bit) {
    if (n <= 1) return launch(type, d, eight_bit, integral_constant<int, 1>{});
    if (n <= 2) return launch(type, d, eight_bit, integral_constant<int, 2>{});
    return launch(type, d, eight_bit, integral_constant<int, 4>{});
  };
  auto with_size = [&](auto type) {
    if (dm.d == 64) return fp8 ? with_rows(type, integral_constant<int, 64>{}, std::true_type{}) : with_rows(type, integral_constant<int, 64>{}, std::false_type{});
    return fp8 ? with_rows(type, integral_constant<int, 128>{}, std::true_type{}) : with_rows(type, integral_constant<int, 128>{}, std::false_type{});
  };
  return dtype == QUOKA_BF16 ? with_size(uint16_t{}) : with_size(float{});
}

}  // namespace quoka
