// tree_attn_mfma.h with changed scores, for bf16 data.
#include "tree_attn_mfma.h"

namespace s4c {

hipError_t launch_tree_attn_large_scored(const AttnArgs& a, int dtype, const score::Args<score::kChanged>& sc, hipStream_t st) {
    return dtype == S4C_F16 ? launch_large_scored_f16(a, sc, st) : launch_large_scored<false>(a, sc, st);
}

}  // namespace s4c
