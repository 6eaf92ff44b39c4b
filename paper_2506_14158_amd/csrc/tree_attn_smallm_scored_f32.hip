// tree_attn_smallm.h with changed scores, for fp32 data.
#include "tree_attn_smallm.h"

namespace s4c {

hipError_t launch_tree_attn_small_scored(const AttnArgs& a, int dtype, const score::Changed& sc, hipStream_t st) {
    return dtype == S4C_F32   ? launch_smallm_scored<kF32>(a, sc, st)
           : dtype == S4C_F16 ? launch_smallm_scored_f16(a, sc, st)
                              : launch_smallm_scored_bf16(a, sc, st);
}

}  // namespace s4c
