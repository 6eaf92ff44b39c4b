// tree_attn_smallm.h with changed scores, for bf16 data.
#include "tree_attn_smallm.h"

namespace s4c {

hipError_t launch_smallm_scored_bf16(const AttnArgs& a, const score::Changed& sc, hipStream_t st) { return launch_smallm_scored<kB16>(a, sc, st); }

}  // namespace s4c
