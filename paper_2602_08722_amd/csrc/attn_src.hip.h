// What an attention kernel over contiguous tensors and one over a cache in pages differ in.
#pragma once
#include <type_traits>

#include "common.hip.h"
#include "kernels.h"
#include "pages.hip.h"

namespace quoka {

// Where the rows of the cache and the chunk lie: in tensors of their own, or in pages, which hold both, as they are or in 8 bits.
constexpr int kContiguous = 0, kRawPages = 1, kFp8Pages = 2;
struct PagedAttnArgs : AttnArgs {   // (n_cache: as in AttnArgs)
  const int32_t *kv_lens = nullptr, *chunk_lens = nullptr;
  Pages pg = {};
  // set by the launcher of the bf16 kernel where lists are shared: blocks of a KV head and their records; row blocks of a block and keys of a
  // tile, as powers of two; number of shares and first record of every KV head's and sequence's list
  u32x2* shares = nullptr;
  int slots = 0, records = 0, block_shift = 0, tile_shift = 0;
};
inline PagedAttnArgs paged_attn_args(const PagedArgs& p, float* part) {
  PagedAttnArgs a;
  a.q = p.q;
  a.k_cache = a.v_cache = a.k_chunk = a.v_chunk = nullptr;
  a.k_idx = p.k_idx;
  a.n_cache = p.k_idx != nullptr ? p.k_cnt : p.kv_lens;
  a.out = p.out;
  a.lse = p.lse;
  a.part = part;
  a.kv_lens = p.kv_lens;
  a.chunk_lens = p.chunk_lens;
  a.pg = p.pg;
  return a;
}
template <int SRC>
using attn_args = std::conditional_t<SRC == kContiguous, AttnArgs, PagedAttnArgs>;
// tokens of batch entry b's chunk
__device__ __forceinline__ int chunk_of(const Dims& dm, const AttnArgs&, int b) { return dm.chunk(b); }
__device__ __forceinline__ int chunk_of(const Dims& dm, const PagedAttnArgs& a, int b) {
  return a.chunk_lens == nullptr ? dm.C : max(min(a.chunk_lens[b], dm.C), 0);
}
// its cached tokens (in pages; elsewhere nothing asks)
__device__ __forceinline__ int paged_len(const Dims&, const AttnArgs&, int) { return 0; }
__device__ __forceinline__ int paged_len(const Dims& dm, const PagedAttnArgs& a, int b) { return min(max(a.kv_lens[b], 0), dm.T_max); }

}  // namespace quoka
