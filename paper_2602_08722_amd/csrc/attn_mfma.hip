// The bf16 attention kernel (attn_mfma.hip.h) over contiguous tensors.
#include "attn_mfma.hip.h"

namespace quoka {

template <int D, bool SPLIT, bool XS>
static hipError_t launch_dsx(const Dims& dm, const AttnArgs& a, hipStream_t st) {
  if (a.n_splits > 1) return launch_variant<D, SPLIT, XS, true, false>(dm, a, st);
  if constexpr (SPLIT) {
    if (dm.g * dm.C < 64) return launch_variant<D, SPLIT, XS, false, false>(dm, a, st);
  }
  return launch_variant<D, SPLIT, XS, false, SPLIT || D == 128>(dm, a, st);
}

template <int D, bool SPLIT>
static hipError_t launch_ds(const Dims& dm, const AttnArgs& a, hipStream_t st) {
  return dm.flags & QUOKA_ATTN_SCALE_F32 ? launch_dsx<D, SPLIT, true>(dm, a, st) : launch_dsx<D, SPLIT, false>(dm, a, st);
}

// Both factors of the first bound grow with the chunk length, so shorter chunks of the same shape fit as well: a prompt's last
// chunk may be split where the others never are (heads * nrb beyond kMaxRecords / 2), with the same workspace.
size_t attn_bf16_ws_floats(const Dims& dm) {
  const long long nrb = (long long)dm.g * ((dm.C + 31) / 32), heads = (long long)dm.n_kv * dm.b;
  const long long most = heads * nrb * key_splits_limit(dm, false, kSub);
  return (size_t)(most < kMaxRecords ? most : kMaxRecords) * 32 * (dm.d + 2);
}

template <int D>
static hipError_t launch_d(const Dims& dm, const AttnArgs& a, hipStream_t st) {
  const AttnPlan p = attn_plan(dm, a.k_idx != nullptr);
  AttnArgs aa = a;
  aa.n_splits = p.n_splits;
  return p.split_tile ? launch_ds<D, true>(dm, aa, st) : launch_ds<D, false>(dm, aa, st);
}

void attn_bf16_plan(const Dims& dm, bool sparse, int32_t* row_blocks, int32_t* n_splits) {
  const AttnPlan p = attn_plan(dm, sparse);
  *row_blocks = p.split_tile ? 4 : 8;
  *n_splits = p.n_splits;
}

hipError_t launch_attn_bf16(const Dims& dm, const AttnArgs& a, float* part, hipStream_t st) {
  AttnArgs aa = a;
  aa.part = part;
  return dm.d == 64 ? launch_d<64>(dm, aa, st) : launch_d<128>(dm, aa, st);
}

}  // namespace quoka
