// Attention of a chunk over a cache in pages: which kernel takes the call.  Float32 attention over pages: the kernel of attn_f32.hip.h, and
// one for short lists.
#include "attn_f32.hip.h"

namespace quoka {

// Short lists of a few tokens, as attn_f32_short: one wave per query row, lanes take 64 keys at a time for the logits and own D / 64
// output dims each for the values.  Bound by a chain of fetches (length, page, rows) and one step a key.  Measured (attn_f32 -> this kernel, rows as
// they are): 32/8 heads, d 128, 1 token over 8 keys 9.2 -> 5.3 us, 8 tokens over 16 9.8 -> 8.3, 1 over 40, the longest, 9.6 -> 10.0; d 64, 1 over 16
// 6.6 -> 6.0; 8-bit pages 10.1 -> 5.6, 10.8 -> 7.9, 7.3 -> 5.8.
constexpr int kPsThreads = 256;

template <bool FP8, int D>
__global__ __launch_bounds__(kPsThreads) void paged_f32_short(Dims dm, PagedArgs a) {
  constexpr int EPL = D / 64;
  __shared__ float qs[kPsThreads / 64][D];
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int i = blockIdx.x * (kPsThreads / 64) + w, h = blockIdx.y, b = blockIdx.z;
  const int C = a.chunk_lens == nullptr ? dm.C : min(a.chunk_lens[b], dm.C);
  const bool row_on = i < C;
  if (row_on) {
    const float* q = static_cast<const float*>(a.q) + b * dm.qs[0] + h * dm.qs[1] + i * dm.qs[2];
#pragma unroll
    for (int e = 0; e < EPL; ++e) qs[w][lane + 64 * e] = q[lane + 64 * e];
  }
  __syncthreads();
  if (!row_on) {   // wave-uniform; no barrier follows
    if (i < dm.C) {   // a row past the sequence's chunk
      float* out = static_cast<float*>(a.out) + b * dm.os[0] + h * dm.os[1] + i * dm.os[2];
#pragma unroll
      for (int e = 0; e < EPL; ++e) out[lane + 64 * e] = 0.f;
      if (a.lse != nullptr && lane == 0) a.lse[(long long)(b * dm.n_q + h) * dm.C + i] = -INFINITY;
    }
    return;
  }
  const int kv = h / dm.g;
  const int n_before = min(max(a.kv_lens[b], 0), dm.T_max);
  const int n_list = a.k_idx == nullptr ? n_before : min(max(a.k_cnt[b * dm.n_kv + kv], 0), dm.B_max);
  const int32_t* list = a.k_idx == nullptr ? nullptr : a.k_idx + (long long)(b * dm.n_kv + kv) * dm.B_max;
  const int32_t* table = pg.table + (long long)b * pg.max_pages;
  const int total = n_list + i + 1;
  const float scale = 1.0f / sqrtf((float)D);
  float m_run = -INFINITY, l_run = 0.f, acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
  for (int j0 = 0; j0 < total; j0 += 64) {
    const int j = min(j0 + lane, total - 1);
    // (the clamp: a malformed list cannot leave the cache)
    const int pos = j >= n_list ? n_before + j - n_list : list == nullptr ? j : (int)min((uint32_t)list[j], (uint32_t)max(dm.T_max - 1, 0));
    const uint32_t page = page_of(pg, table, pos);
    const long long row = row_at(pg, page, kv, slot_of(pg, pos)), row_scale_at = scale_at(pg, page, kv, slot_of(pg, pos));
    const float ks = FP8 ? row_scale(pg.k_scale[row_scale_at]) : 1.f, vs = FP8 ? row_scale(pg.v_scale[row_scale_at]) : 1.f;
    float dot = 0.f;
#pragma unroll 4
    for (int d0 = 0; d0 < D; d0 += 8) {
      float x[8];
      if constexpr (FP8) {
        const u32x2 x8 = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pg.k) + row + d0);
        widen_f32(x8[0], ks, x);
        widen_f32(x8[1], ks, x + 4);
      } else {
        Elem<float>::load8(static_cast<const float*>(pg.k) + row + d0, x);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += qs[w][d0 + e] * x[e];
    }
    const bool valid = j0 + lane < total;
    const float s = valid ? dot * scale : -INFINITY;
    const float m_new = fmaxf(m_run, wave64_max(s));   // finite: key j0 is always visible
    const float alpha = expf(m_run - m_new), p = valid ? expf(s - m_new) : 0.f;
    l_run = l_run * alpha + wave64_sum(p);
    m_run = m_new;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] *= alpha;
    const int n = min(64, total - j0);
    for (int t = 0; t < n; ++t) {   // t is wave-uniform: lane reads through the scalar path
      const float pt = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), t));
      const float vt = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs), t));
      const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)row, t), hi = (uint32_t)__builtin_amdgcn_readlane((int)(row >> 32), t);
      const long long at = (long long)((uint64_t)hi << 32 | lo) + lane;
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        if constexpr (FP8) acc[e] += pt * (__builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(pg.v)[at + 64 * e], 0) * vt);
        else acc[e] += pt * static_cast<const float*>(pg.v)[at + 64 * e];
      }
    }
  }
  float* out = static_cast<float*>(a.out) + b * dm.os[0] + h * dm.os[1] + i * dm.os[2];
#pragma unroll
  for (int e = 0; e < EPL; ++e) out[lane + 64 * e] = acc[e] / l_run;
  if (a.lse != nullptr && lane == 0) a.lse[(long long)(b * dm.n_q + h) * dm.C + i] = m_run + logf(l_run);
}

template <bool FP8, int D>
static hipError_t launch_paged_f32(const Dims& dm, const PagedArgs& a, float* part, hipStream_t st) {
  if (attn_f32_is_short(dm, a.k_idx != nullptr)) {
    const dim3 grid((dm.C + kPsThreads / 64 - 1) / (kPsThreads / 64), dm.n_q, dm.b);
    hipLaunchKernelGGL((paged_f32_short<FP8, D>), grid, dim3(kPsThreads), 0, st, dm, a);
    return hipGetLastError();
  }
  return launch_f32_units<D, FP8 ? kFp8Pages : kRawPages>(dm, paged_attn_args(a, part), part, st);
}

size_t paged_attn_ws_floats(const Dims& dm, int dtype) {
  if (dtype != QUOKA_BF16) return attn_f32_ws_floats(dm);
  return attn_decode_applies(dm) ? paged_decode_ws_floats(dm) : paged_attn_bf16_ws_floats(dm);
}

hipError_t launch_paged_attn(const Dims& dm, int dtype, bool fp8, const PagedArgs& a, float* part, hipStream_t st) {
  if (dtype == QUOKA_BF16)
    return attn_decode_applies(dm) ? launch_paged_decode(dm, fp8, a, part, st) : launch_paged_attn_bf16(dm, fp8, a, part, st);
  if (dm.d == 64) return fp8 ? launch_paged_f32<true, 64>(dm, a, part, st) : launch_paged_f32<false, 64>(dm, a, part, st);
  return fp8 ? launch_paged_f32<true, 128>(dm, a, part, st) : launch_paged_f32<false, 128>(dm, a, part, st);
}

}  // namespace quoka
