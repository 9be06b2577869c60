// Rows of a cache in pages into other pages, as they are kept (quoka_cache_copy, quoka_cache_compact).
//
// Bound by memory: every row is read once and written once.  A row is CG lanes of 16 bytes; a thread has U rows of K and of V on the way at
// once, and the chain ahead of them is length (or list), both pages, row.  Measured, caches that are in no cache memory: lists of 8192 for each
// of 4 sequences and 8 heads of 128, 16-bit rows (269 MB read and written) 56 us (4.8 TB/s; a copy of 1 GiB on this card 5.1), 8-bit rows 27.8 (4.9);
// 333 of 3 sequences and 3 float32 heads of 64 3.5, of which launch and chain are all.
#include <type_traits>

#include "pages.hip.h"

namespace quoka {

constexpr int kPrThreads = 256;

// LIST (compact): row i of a list is the row at position list[i] and goes to position i.  Otherwise (copy) row i is that at position
// first + i of the parent, and keeps its position.  Pages' strides come in bytes here.
template <int CG, bool FP8, bool LIST, int U>
__global__ __launch_bounds__(kPrThreads) void move_rows(MoveArgs a) {
  constexpr int RPB = kPrThreads / CG;
  const int kv = (int)blockIdx.y % a.n_kv, b = (int)blockIdx.y / a.n_kv;
  const int r0 = threadIdx.x / CG, c = threadIdx.x % CG;
  const int i0 = (int)blockIdx.x * RPB * U;
  int n, first = 0, from = b;
  const int32_t* list = nullptr;
  if constexpr (LIST) {
    n = min(a.cnt[b * a.n_kv + kv], a.B_max);
    list = a.list + (long long)(b * a.n_kv + kv) * a.B_max;
  } else {
    first = a.first == nullptr ? 0 : max(a.first[b], 0);
    from = a.parents == nullptr ? b : a.parents[b];
    n = min(max(a.lens[b], 0) - first, a.max_rows);
    if ((uint32_t)from >= (uint32_t)a.n_parents) return;   // block-uniform
  }
  if (i0 >= n) return;   // block-uniform
  const int32_t* src_table = a.src.table + (long long)from * a.src.max_pages;
  const int32_t* dst_table = a.dst.table + (long long)b * a.dst.max_pages;
  uint32_t pos[U], src_page[U], dst_page[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = min(i0 + u * RPB + r0, n - 1);
    // (the clamp: a malformed list cannot leave the cache)
    pos[u] = LIST ? min((uint32_t)list[i], (uint32_t)max(a.T_max - 1, 0)) : (uint32_t)(first + i);
    dst_page[u] = (uint32_t)dst_table[min((LIST ? i : first + i) >> a.dst.shift, a.dst.max_pages - 1)];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t at = pos[u] >> a.src.shift;
    src_page[u] = (uint32_t)src_table[min(at, (uint32_t)a.src.max_pages - 1)];
    // (no page in either: the row is dropped; what is fetched in its place is inside the pool)
    if (src_page[u] >= (uint32_t)a.src.n_pages || at >= (uint32_t)a.src.max_pages) dst_page[u] = ~0u, src_page[u] = 0;
  }
  u32x4 xk[U], xv[U];
  uint8_t ek[FP8 ? U : 1], ev[FP8 ? U : 1];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int slot = slot_of(a.src, (int)pos[u]);
    const long long at = row_at(a.src, src_page[u], kv, slot) + 16 * c;
    xk[u] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.src.k) + at);
    xv[u] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.src.v) + at);
    if constexpr (FP8) {
      const long long s = scale_at(a.src, src_page[u], kv, slot);
      ek[u] = a.src.k_scale[s];
      ev[u] = a.src.v_scale[s];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = i0 + u * RPB + r0, to = LIST ? i : first + i;
    if (i >= n || dst_page[u] >= (uint32_t)a.dst.n_pages || (to >> a.dst.shift) >= a.dst.max_pages) continue;
    const int slot = slot_of(a.dst, to);
    const long long at = row_at(a.dst, dst_page[u], kv, slot) + 16 * c;
    u32x4 *to_k = reinterpret_cast<u32x4*>(static_cast<char*>(a.dst.k) + at), *to_v = reinterpret_cast<u32x4*>(static_cast<char*>(a.dst.v) + at);
    if constexpr (LIST) {   // (past the cache memories, which long lists would fill: 59.6 -> 56.4 us and 33.3 -> 27.8 in the two cases above)
      __builtin_nontemporal_store(xk[u], to_k);
      __builtin_nontemporal_store(xv[u], to_v);
    } else {
      *to_k = xk[u];
      *to_v = xv[u];
    }
    if constexpr (FP8) {
      const long long s = scale_at(a.dst, dst_page[u], kv, slot);
      if (c == 0) {
        a.dst.k_scale[s] = ek[u];
        a.dst.v_scale[s] = ev[u];
      }
    }
  }
}

hipError_t launch_move_rows(MoveArgs a, int batch, int row_bytes, bool fp8, hipStream_t st) {
  constexpr int U = 2;   // (1, 2, 4: 59.4, 59.6, 60.7 us and 33.5, 33.3, 33.4)
  for (int i = 0; i < 3; ++i) {
    a.src.st[i] *= a.es;
    a.dst.st[i] *= a.es;
  }
  const int most = a.list != nullptr ? a.B_max : a.max_rows;
  if (most <= 0) return hipSuccess;
  auto launch = [&](auto chunks, auto eight_bit) {
    constexpr int CG = decltype(chunks)::value, ROWS = kPrThreads / CG * U;
    constexpr bool FP8 = decltype(eight_bit)::value;
    const dim3 grid((most + ROWS - 1) / ROWS, batch * a.n_kv);
    if (a.list != nullptr) hipLaunchKernelGGL((move_rows<CG, FP8, true, U>), grid, dim3(kPrThreads), 0, st, a);
    else hipLaunchKernelGGL((move_rows<CG, FP8, false, U>), grid, dim3(kPrThreads), 0, st, a);
    return hipGetLastError();
  };
  using std::integral_constant;
  if (fp8) return row_bytes == 64 ? launch(integral_constant<int, 4>{}, std::true_type{}) : launch(integral_constant<int, 8>{}, std::true_type{});
  switch (row_bytes) {
    case 128: return launch(integral_constant<int, 8>{}, std::false_type{});
    case 256: return launch(integral_constant<int, 16>{}, std::false_type{});
    default: return launch(integral_constant<int, 32>{}, std::false_type{});
  }
}

}  // namespace quoka
