// The bf16 attention kernel (attn_mfma.hip.h) over states in pages (quoka_cross_attn): every query sees all of its sequence's cached rows.
//
// Without a mask all row blocks of a launch take equally long, and the tiles are those of the list alone.
// Bound by matrix and vector instructions together (matrix units 60 % busy at the clock it runs at).  Measured: 2048 tokens over 16384 states, 32/8 heads
// of 128, 474 - 486 us on four cards (1.13 - 1.16 PFLOP/s; a large matrix product reaches 1.36).
#include "attn_mfma.hip.h"

namespace quoka {

template <int D, bool SPLIT, int SRC>
static hipError_t launch_states_ds(const Dims& dm, const PagedAttnArgs& a, hipStream_t st) {
  if (a.n_splits > 1) return launch_variant<D, SPLIT, true, true, false, SRC>(dm, a, st);
  return launch_variant<D, SPLIT, true, false, SPLIT || D == 128, SRC>(dm, a, st);
}

hipError_t launch_cross_attn_bf16(const Dims& dm, bool fp8, const PagedArgs& a, float* part, hipStream_t st) {
  const AttnPlan p = attn_plan(dm, false, true, false);
  PagedAttnArgs aa = paged_attn_args(a, part);
  aa.n_splits = p.n_splits;
  aa.shares = reinterpret_cast<u32x2*>(part + attn_bf16_ws_floats(dm));   // (behind all partials)
  auto launch = [&](auto d, auto src) {
    constexpr int D = decltype(d)::value, SRC = decltype(src)::value;
    return p.split_tile ? launch_states_ds<D, true, SRC>(dm, aa, st) : launch_states_ds<D, false, SRC>(dm, aa, st);
  };
  using d64 = std::integral_constant<int, 64>;
  using d128 = std::integral_constant<int, 128>;
  using raw = std::integral_constant<int, kRawStates>;
  using eight_bit = std::integral_constant<int, kFp8States>;
  if (dm.d == 64) return fp8 ? launch(d64{}, eight_bit{}) : launch(d64{}, raw{});
  return fp8 ? launch(d128{}, eight_bit{}) : launch(d128{}, raw{});
}

}  // namespace quoka
