// Changed scores of the attention kernels (s4c_tree_attn_scored) and the log-sum-exp of a row.
//
//   x = scale q.k;   cap > 0: x <- cap tanh(x / cap);   slopes: x <- x + slope[head] (position of the key - position of the root)
//
// In log2 units throughout.  The distance is counted from the root and not from the row's node: the difference is the same for all
// keys of a row, and the softmax does not see it.  Positions are differences of 32-bit integers first and fp32 after: exact up to 2^24.
//
// What it costs is operations of the vector ALUs, of which a score otherwise has about eight (four of them its exponential):
//   bias              for many rows none: an fp32 product of the keys' distances and the rows' slopes is added by the matrix cores, 64 cycles for 32 x 32
//                     scores (slopes are divided by the scale once, so that it goes to the bare products).  For few rows, where a wave waits for that, one
//                     by rows (the tile's own distance goes to the reference of the exponentials), three where positions are looked up.  The one and the
//                     other, us: 16 x 64/8 heads, 32768 keys + 128 nodes, looked up 2105 and 2200; 13 x 32/8 heads, 5003 keys, one node 28.6 and 25.1
//   cap               C y p(y^2), y = x / cap, C = cap log2(e), p a fit of tanh(y)/y at Chebyshev nodes.  Where all scores of a wave are within 0.35
//                     of the cap (and nothing is added), the kernel for many rows takes four terms (relative error 3.5e-8) with the scale in the
//                     coefficients, and the last product is the one that makes the exponent: four more operations.  Within 0.6 five
//                     terms (7.5e-8).  Beyond, C - 2 C / (1 + exp2(2 log2(e) |y|)) with y's sign, two more operations at a quarter of the rate, off by
//                     C 2^-23, a relative 2.2e-7 there.
#pragma once
#include "common.h"

#include "attn_parts.h"

namespace s4c {
namespace score {

using mfma::f32x16;
using mfma::f32x4;
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr float kFitUpTo = 0.6f;
constexpr float kFit[5] = {0.99999993f, -0.33332323f, 0.13310358f, -0.05210962f, 0.01548669f};

// tanh(y), |y| <= kFitUpTo, times c
__device__ __forceinline__ float fitted(float y, float c) {
    const float z = y * y;
    float p = fmaf(z, kFit[4] * c, kFit[3] * c);
    p = fmaf(z, p, kFit[2] * c);
    p = fmaf(z, p, kFit[1] * c);
    p = fmaf(z, p, kFit[0] * c);
    return y * p;
}
// (of |y|, and y's sign put back: below 0 the quotient would be the larger part of the result, with three times the rounding)
__device__ __forceinline__ float beyond(float y, float c) {
    const float e = fast_exp2(fabsf(y) * (2.f * kLog2e));       // infinity: the cap
    return copysignf(fmaf(-2.f * c, __builtin_amdgcn_rcpf(1.f + e), c), y);
}

// products -> c tanh(to_y product) (cap > 0); N values, s(j) a reference to the j-th
template <int N, class V>
__device__ __forceinline__ void cap_all(V s, const Changed& a, float c) {
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        s(j) *= a.to_y;
        most = fmaxf(most, fabsf(s(j)));
    }
    if (!__any(most > kFitUpTo)) {
#pragma unroll
        for (int j = 0; j < N; ++j) s(j) = fitted(s(j), c);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) s(j) = fabsf(s(j)) <= kFitUpTo ? fitted(s(j), c) : beyond(s(j), c);
    }
}
// ... of a tile of 32 keys (a lane's register j), and of NG blocks of 16 x 16
__device__ __forceinline__ void cap(f32x16& s, const Changed& a, float c) {
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = s[j];
    cap_all<16>([&](int j) -> float& { return x[j]; }, a, c);
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = x[j];
}
template <int NG>
__device__ __forceinline__ void cap(f32x4 (&s)[NG], const Changed& a, float c) {
    float x[4 * NG];
#pragma unroll
    for (int j = 0; j < 4 * NG; ++j) x[j] = s[j >> 2][j & 3];
    cap_all<4 * NG>([&](int j) -> float& { return x[j]; }, a, c);
#pragma unroll
    for (int j = 0; j < 4 * NG; ++j) s[j >> 2][j & 3] = x[j];
}
// What a value of a tile is multiplied with to be a score in log2 units.  FIT: a product within fit_up_to is capped by it, s p(s^2) in
// all; one that is a tanh already is multiplied by the cap with the same instructions, so that one line of code lies behind the choice (a tanh, and
// not what it is multiplied to: that one's square can be infinite).
template <bool FIT>
struct Factor {
    float c[4];
    __device__ __forceinline__ Factor(const Changed& a, bool fits, float)
        : c{fits ? a.fit[0] : a.cap_log2, fits ? a.fit[1] : 0.f, fits ? a.fit[2] : 0.f, fits ? a.fit[3] : 0.f} {}
    __device__ __forceinline__ float operator()(float s) const {
        const float z = s * s;
        return fmaf(z, fmaf(z, fmaf(z, c[3], c[2]), c[1]), c[0]);
    }
};
template <>
struct Factor<false> {
    float mul;
    template <class Score>
    __device__ __forceinline__ Factor(const Score&, bool, float m) : mul(m) {}
    __device__ __forceinline__ float operator()(float) const { return mul; }
};

// The bias of a block of 32 keys and 32 rows is the product of a column and a row, which the matrix cores add: `distance` is the position of key
// lane % 32 from the root's, `slope` that of row lane % 32 (the instruction's second term is 0).
__device__ __forceinline__ f32x16 add_bias(float distance, float slope, const f32x16& s) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32((threadIdx.x & 32) == 0 ? distance : 0.f, slope, s, 0, 0, 0);
}
// The same by the vector ALUs.  Register j of a lane is key 8 (j/4) + j%4 of the lane's part of a block.
// ... whose first key is row `first` before (< 0) or behind the root; returns what is left to add to the lane's scores, in log2 units.
// (Counted from the part's last key, the one next to the root: there the sums are small, and so are their roundings.)
__device__ __forceinline__ float add_rows(f32x16& s, float slope, int first, const Changed& a) {
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = fmaf((float)(8 * (j >> 2) + (j & 3) - 27), slope, s[j]);
    return slope * a.mul * (float)(first + 27);
}
// ... whose positions lie in LDS
__device__ __forceinline__ void add_looked_up(f32x16& s, float slope, const int32_t* pos, int root) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const i32x4 p = *(const i32x4*)(pos + 8 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * q + e] = fmaf(slope, (float)(p[e] - root), s[4 * q + e]);
    }
}
// ... of nodes of the tree
__device__ __forceinline__ void add_depths(f32x16& s, float slope, const float* depth) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x4 d = *(const f32x4*)(depth + 8 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * q + e] = fmaf(slope, d[e], s[4 * q + e]);
    }
}
// every node's depth, by the thread that has written its ancestors
__device__ __forceinline__ void note_depth(const AttnArgs& a, const uint32_t* anc, float* depth) {
    const int i = threadIdx.x;
    if (i < a.N) {
        const uint4 m = *(const uint4*)(anc + 4 * i);
        depth[i] = (float)(__popc(m.x) + __popc(m.y) + __popc(m.z) + __popc(m.w) - 1);
    }
}

// Writes a row's log-sum-exp (natural) from its reference m (log2 units) and sum l of 2^(x - m + shift); a row without any (a flagged
// sequence) has +infinity, so that exp(x - lse) is 0.
struct Writer {
    float* lse;
    float shift;
    __device__ __forceinline__ void operator()(size_t row, float m, float l) const {
        if (lse) lse[row] = l > 0.f ? (m - shift + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : INFINITY;
    }
};
__device__ __forceinline__ work::NoRowDone writer(const Unchanged&, float) { return {}; }
__device__ __forceinline__ Writer writer(const Changed& a, float shift) { return {a.lse, shift}; }

}  // namespace score
}  // namespace s4c
