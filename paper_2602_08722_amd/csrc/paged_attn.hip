// Attention of a chunk over a cache in pages (quoka_paged_attn): one wave a query row, 64 keys at a time.
#include "pages.hip.h"

namespace quoka {

constexpr int kPaThreads = 256;

template <typename T, bool FP8>
__device__ __forceinline__ void load_row8(const void* pages, long long row, int e0, float scale, float (&x)[8]) {
  if constexpr (FP8) {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pages) + row + e0);
    widen_f32(w.x, scale, x);
    widen_f32(w.y, scale, x + 4);
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
  const int total = i < C ? n_list + i + 1 : 0;
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
    const float o = total > 0 ? acc[e] / l_run : 0.f;
    if constexpr (sizeof(T) == 2) out[lane + 64 * e] = (T)f32_to_bf16_bits(o);
    else out[lane + 64 * e] = o;
  }
  if (a.lse != nullptr && lane == 0) a.lse[(long long)(b * dm.n_q + h) * dm.C + i] = total > 0 ? m_run + logf(l_run) : -INFINITY;
}

size_t paged_attn_ws_floats(const Dims&, int) { return 0; }

hipError_t launch_paged_attn(const Dims& dm, int dtype, bool fp8, const PagedArgs& a, float*, hipStream_t st) {
  const dim3 grid((dm.C + 3) / 4, dm.n_q, dm.b);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kPaThreads), 0, st, dm, a);
    return hipGetLastError();
  };
  if (dtype == QUOKA_BF16) {
    if (dm.d == 64) return fp8 ? launch(paged_attn_rows<uint16_t, true, 64>) : launch(paged_attn_rows<uint16_t, false, 64>);
    return fp8 ? launch(paged_attn_rows<uint16_t, true, 128>) : launch(paged_attn_rows<uint16_t, false, 128>);
  }
  if (dm.d == 64) return fp8 ? launch(paged_attn_rows<float, true, 64>) : launch(paged_attn_rows<float, false, 64>);
  return fp8 ? launch(paged_attn_rows<float, true, 128>) : launch(paged_attn_rows<float, false, 128>);
}

}  // namespace quoka
