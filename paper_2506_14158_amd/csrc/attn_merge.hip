// The merge kernel of a divided attention launch (attn_merge.h), as a launch of its own.
#include "attn_merge.h"
#include "attn_score.h"

namespace s4c {

namespace {

template <typename T, int D, class Score>
__global__ __launch_bounds__(256) void attn_merge_kernel(AttnArgs a, int passes, Score sc) {
    constexpr float kShift = std::is_same<T, float>::value ? 0.f : mfma::Prob<std::is_same<T, f16_t>::value, D>::kShift;
    merge::merge_rows<T, D>(a, blockIdx.x, blockIdx.y, passes, score::writer(sc, kShift));
}

template <typename T, class Score>
hipError_t launch(const AttnArgs& a, const Score& sc, hipStream_t st) {
    const merge::Grid g = merge::grid_of(a);
    const dim3 grid((unsigned)g.units, (unsigned)g.chunks), block(256);
    if (a.D == 64) hipLaunchKernelGGL((attn_merge_kernel<T, 64, Score>), grid, block, 0, st, a, g.passes, sc);
    else hipLaunchKernelGGL((attn_merge_kernel<T, 128, Score>), grid, block, 0, st, a, g.passes, sc);
    return hipGetLastError();
}
template <class Score>
hipError_t launch(const AttnArgs& a, int dtype, const Score& sc, hipStream_t st) {
    return dtype == S4C_F32 ? launch<float>(a, sc, st) : dtype == S4C_F16 ? launch<f16_t>(a, sc, st) : launch<bf16_t>(a, sc, st);
}

}  // namespace

hipError_t launch_attn_merge(const AttnArgs& a, int dtype, hipStream_t st) { return launch(a, dtype, score::Unchanged(), st); }
hipError_t launch_attn_merge(const AttnArgs& a, int dtype, const score::Changed& sc, hipStream_t st) { return launch(a, dtype, sc, st); }

}  // namespace s4c
