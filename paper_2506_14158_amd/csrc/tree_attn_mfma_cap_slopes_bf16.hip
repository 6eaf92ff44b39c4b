// tree_attn_mfma.h for bf16 data, with capped scores and slopes over the keys' positions.
#include "tree_attn_mfma.h"

namespace s4c {

hipError_t launch_large_cap_slopes_bf16(const AttnArgs& a, const score::Changed& sc, hipStream_t st) { return launch_large_scored<false, score::kCapSlopes>(a, sc, st); }

}  // namespace s4c
