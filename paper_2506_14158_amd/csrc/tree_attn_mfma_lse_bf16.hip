// tree_attn_mfma.h for bf16 data, with no change to its scores but the log-sum-exp of every row; and the choice between the kinds.
#include "tree_attn_mfma.h"

namespace s4c {

hipError_t launch_large_lse_bf16(const AttnArgs& a, const score::Changed& sc, hipStream_t st) { return launch_large_scored<false, score::kLse>(a, sc, st); }

// The kernel for a cap alone takes the difference of the cap's last product and the reference without rounding the product, as the reference was:
// half a step of a score too much or too little in an exponent, which must not be large.  The one with a bias rounds both.
constexpr float kWide = 0x1p20f;

hipError_t launch_tree_attn_large_scored(const AttnArgs& a, int dtype, const score::Changed& sc, hipStream_t st) {
    if (sc.cap_log2 > 0.f && (sc.slopes || sc.cap_log2 > kWide)) return dtype == S4C_F16 ? launch_large_cap_slopes_f16(a, sc, st) : launch_large_cap_slopes_bf16(a, sc, st);
    if (sc.cap_log2 > 0.f) return dtype == S4C_F16 ? launch_large_cap_f16(a, sc, st) : launch_large_cap_bf16(a, sc, st);
    if (sc.slopes) return dtype == S4C_F16 ? launch_large_slopes_f16(a, sc, st) : launch_large_slopes_bf16(a, sc, st);
    return dtype == S4C_F16 ? launch_large_lse_f16(a, sc, st) : launch_large_lse_bf16(a, sc, st);
}

}  // namespace s4c
