// The bf16 attention kernel (attn_mfma.hip.h) over a cache in pages.
#include "attn_mfma.hip.h"

namespace quoka {

template <int D, bool SPLIT, int SRC>
static hipError_t launch_paged_ds(const Dims& dm, const PagedAttnArgs& a, hipStream_t st) {
  if (a.n_splits > 1) return launch_variant<D, SPLIT, true, true, false, SRC>(dm, a, st);
  return launch_variant<D, SPLIT, true, false, SPLIT || D == 128, SRC>(dm, a, st);
}

size_t paged_attn_bf16_ws_floats(const Dims& dm) { return attn_bf16_ws_floats(dm) + (size_t)2 * dm.n_kv * dm.b; }

hipError_t launch_paged_attn_bf16(const Dims& dm, bool fp8, const PagedArgs& a, float* part, hipStream_t st) {
  const AttnPlan p = attn_plan(dm, a.k_idx != nullptr, true);
  PagedAttnArgs aa = paged_attn_args(a, part);
  aa.n_splits = p.n_splits;
  aa.shares = reinterpret_cast<u32x2*>(part + attn_bf16_ws_floats(dm));   // (behind all partials)
  auto launch = [&](auto d, auto src) {
    constexpr int D = decltype(d)::value, SRC = decltype(src)::value;
    return p.split_tile ? launch_paged_ds<D, true, SRC>(dm, aa, st) : launch_paged_ds<D, false, SRC>(dm, aa, st);
  };
  using d64 = std::integral_constant<int, 64>;
  using d128 = std::integral_constant<int, 128>;
  using raw = std::integral_constant<int, kRawPages>;
  using eight_bit = std::integral_constant<int, kFp8Pages>;
  if (dm.d == 64) return fp8 ? launch(d64{}, eight_bit{}) : launch(d64{}, raw{});
  return fp8 ? launch(d128{}, eight_bit{}) : launch(d128{}, raw{});
}

}  // namespace quoka
