// tree_attn_mfma.h for fp16 data, with no change to its scores but the log-sum-exp of every row.
#include "tree_attn_mfma.h"

namespace s4c {

hipError_t launch_large_lse_f16(const AttnArgs& a, const score::Changed& sc, hipStream_t st) { return launch_large_scored<true, score::kLse>(a, sc, st); }

}  // namespace s4c
