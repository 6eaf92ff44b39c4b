// tree_attn_mfma.h with changed scores, for fp16 data.
#include "tree_attn_mfma.h"

namespace s4c {

hipError_t launch_large_scored_f16(const AttnArgs& a, const score::Args<score::kChanged>& sc, hipStream_t st) { return launch_large_scored<true>(a, sc, st); }

}  // namespace s4c
