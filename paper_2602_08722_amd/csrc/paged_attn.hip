// Attention of a chunk over a cache in pages (quoka_paged_attn): one wave a query row, 64 keys at a time.
#include "pages.hip.h"

namespace quoka {

constexpr int kPaThreads = 256;

template <typename T, bool FP8>
__device__ __forceinline__ void load_row8(const void* pages, long long row, int e0, float scale, float (&x)[8]) {
  if constexpr (FP8) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pages) + row + e0);
    widen_f32(w[0], scale, x);
    widen_f32(w[1], scale, x + 4);
  } else {
    Elem<T>::load8(static_cast<const T*>(pages) + row + e0, x);
  }
}

template <typename T, bool FP8, int D>
__global__ __launch_bounds__(kPaThreads) void paged_attn_rows(Dims dm, PagedArgs a) {
  constexpr int EPL = D / 64;
  __shared__ float qs[kPaThreads / 64][D];
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int i = blockIdx.x * (kPaThreads / 64) + w, h = blockIdx.y, b = blockIdx.z;
  const bool row_on = i < dm.C;
  if (row_on) {
    const T* q = static_cast<const T*>(a.q) + b * dm.qs[0] + h * dm.qs[1] + i * dm.qs[2];
#pragma unroll
    for (int e = 0; e < EPL; ++e) qs[w][lane + 64 * e] = Elem<T>::load1(q + lane + 64 * e);
  }
  __syncthreads();
  if (!row_on) return;
  const int kv = h / dm.g;
  const int C = a.chunk_lens == nullptr ? dm.C : min(a.chunk_lens[b], dm.C);
  const int T_b = min(max(a.kv_lens[b], 0), dm.T_max);
  const int n_list = a.k_idx == nullptr ? T_b : min(max(a.k_cnt[b * dm.n_kv + kv], 0), dm.B_max);
  const int32_t* list = a.k_idx == nullptr ? nullptr : a.k_idx + (long long)(b * dm.n_kv + kv) * dm.B_max;
  const int32_t* table = pg.table + (long long)b * pg.max_pages;
  if (i >= C) return;
  const int total = n_list + i + 1;
  const float scale = 1.0f / sqrtf((float)D);
  float m_run = -INFINITY, l_run = 0.f, acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
  for (int j0 = 0; j0 < total; j0 += 64) {
    const int j = min(j0 + lane, total - 1);
    const int pos = j < n_list ? (list == nullptr ? j : (int)min((uint32_t)list[j], (uint32_t)max(dm.T_max - 1, 0))) : T_b + j - n_list;
    const uint32_t page = page_of(pg, table, pos);
    const long long row = row_at(pg, page, kv, slot_of(pg, pos)), srow = scale_at(pg, page, kv, slot_of(pg, pos));
    const float ks = FP8 ? row_scale(pg.k_scale[srow]) : 1.f, vs = FP8 ? row_scale(pg.v_scale[srow]) : 1.f;
    float dot = 0.f;
    for (int e0 = 0; e0 < D; e0 += 8) {
      float x[8];
      load_row8<T, FP8>(pg.k, row, e0, ks, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += qs[w][e0 + e] * x[e];
    }
    const bool valid = j0 + lane < total;
    const float s = valid ? dot * scale : -INFINITY;
    const float m_new = fmaxf(m_run, wave64_max(s));
    const float alpha = expf(m_run - m_new), p = valid ? expf(s - m_new) : 0.f;
    l_run = l_run * alpha + wave64_sum(p);
    m_run = m_new;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] *= alpha;
    const int n = min(64, total - j0);
    for (int t = 0; t < n; ++t) {
      const float pt = __shfl(p, t, 64), st = __shfl(vs, t, 64);
      const long long rt = __shfl(row, t, 64);
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        float x;
        if constexpr (FP8) {
          x = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(pg.v)[rt + lane + 64 * e], 0) * st;
        } else {
          x = Elem<T>::load1(static_cast<const T*>(pg.v) + rt + lane + 64 * e);
        }
        acc[e] += pt * x;
      }
    }
  }
  T* out = static_cast<T*>(a.out) + b * dm.os[0] + h * dm.os[1] + i * dm.os[2];
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    const float o = acc[e] / l_run;
    if constexpr (sizeof(T) == 2) out[lane + 64 * e] = (T)f32_to_bf16_bits(o);
    else out[lane + 64 * e] = o;
  }
  if (a.lse != nullptr && lane == 0) a.lse[(long long)(b * dm.n_q + h) * dm.C + i] = m_run + logf(l_run);
}

// Rows past a sequence's chunk: zeros, and no weight at all.  (A launch of its own, and only where lengths are given, since the attention
// kernels' grids follow the chunk's row blocks and such rows may be most of a ragged batch.)
constexpr int kFillRows = 32;
__global__ __launch_bounds__(256) void paged_fill(Dims dm, PagedArgs a, int row_units) {   // row_units: 16-byte units of a row
  const int h = blockIdx.y, b = blockIdx.z, C = max(min(a.chunk_lens[b], dm.C), 0);
  const int i0 = max((int)blockIdx.x * kFillRows, C), i1 = min((int)(blockIdx.x + 1) * kFillRows, dm.C);
  const long long es = dm.d * 2 == row_units * 16 ? 2 : 4;
  char* out = static_cast<char*>(a.out) + (b * dm.os[0] + h * dm.os[1]) * es;
  for (int u = threadIdx.x; u < (i1 - i0) * row_units; u += 256)
    *reinterpret_cast<u32x4*>(out + (i0 + u / row_units) * dm.os[2] * es + (u % row_units) * 16) = u32x4{0u, 0u, 0u, 0u};
  if (a.lse != nullptr)
    for (int i = i0 + threadIdx.x; i < i1; i += 256) a.lse[(long long)(b * dm.n_q + h) * dm.C + i] = -INFINITY;
}

size_t paged_attn_ws_floats(const Dims& dm, int dtype) {
  if (dtype != QUOKA_BF16) return 0;
  return attn_decode_applies(dm) ? paged_decode_ws_floats(dm) : attn_bf16_ws_floats(dm);
}

hipError_t launch_paged_attn(const Dims& dm, int dtype, bool fp8, const PagedArgs& a, float* part, hipStream_t st) {
  if (a.chunk_lens != nullptr) {
    hipLaunchKernelGGL(paged_fill, dim3((dm.C + kFillRows - 1) / kFillRows, dm.n_q, dm.b), dim3(256), 0, st, dm, a,
                       dm.d * (dtype == QUOKA_BF16 ? 2 : 4) / 16);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (dtype == QUOKA_BF16)
    return attn_decode_applies(dm) ? launch_paged_decode(dm, fp8, a, part, st) : launch_paged_attn_bf16(dm, fp8, a, part, st);
  const dim3 grid((dm.C + 3) / 4, dm.n_q, dm.b);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kPaThreads), 0, st, dm, a);
    return hipGetLastError();
  };
  if (dm.d == 64) return fp8 ? launch(paged_attn_rows<float, true, 64>) : launch(paged_attn_rows<float, false, 64>);
  return fp8 ? launch(paged_attn_rows<float, true, 128>) : launch(paged_attn_rows<float, false, 128>);
}

}  // namespace quoka
