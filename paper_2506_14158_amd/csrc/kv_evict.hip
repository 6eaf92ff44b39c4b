// A cache cut down to a budget (s4c_kv_evict): of every (layer, sequence, KV head) the most recent rows stay, and of the others those
// with the largest totals of attention weight (equal ones: lowest row first), `budget` rows altogether.
//
// Rows that stay and lie behind the budget move into the places that evicted rows leave before it, the i-th into the i-th: every source
// lies behind the budget and every place before it, so rows move in any order, in place, and no more of them than must.  (Attention does
// not ask for an order of the keys; what depends on a row's age reads its position.)
//
// Two launches.  evict_select_kernel, a workgroup per unit, finds the smallest key that stays by a radix descent (histograms of 11, 11 and
// 10 bits; a key is the total's bits in integer order, all ones for recent rows) and lists places and movers in row order.
// evict_move_kernel copies the rows: bound by the memory.
#include "common.h"

namespace s4c {

namespace {

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;
constexpr int kBins = 2048, kCopies = 4;
constexpr int kMove = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    return x;
}

// a total's bits in the order of the numbers, below all ones; -0 as 0
__device__ __forceinline__ uint32_t key_of(float w, bool recent) {
    const uint32_t u = __float_as_uint(w + 0.f);
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return recent ? 0xFFFFFFFFu : k < 0xFFFFFFFEu ? k : 0xFFFFFFFEu;
}

__global__ __launch_bounds__(kSelect) void evict_select_kernel(EvictArgs a) {
    __shared__ uint32_t hist[kCopies][kBins];
    __shared__ uint32_t s_wave[4][kSelectWaves];
    __shared__ uint32_t s_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int unit = blockIdx.x, b = (unit / a.Hkv) % a.B;
    const int n = a.cache_len[b];
    bool bad = n < 0 || n > a.S_cap;
    if (!bad && a.block_table)
        for (int i = tid; i < (n + (1 << a.page_shift) - 1) >> a.page_shift; i += kSelect) {
            const int id = a.block_table[(size_t)b * a.max_blocks + i];
            bad = bad || id < 0 || id >= a.num_pages;
        }
    bad = __syncthreads_or(bad) != 0;
    const int m = min(n, a.budget);
    const size_t row0 = (size_t)unit * a.S_cap;
    const float* w = a.weight + row0;
    const int32_t* pos = a.key_pos + row0;
    int32_t* kept = a.kept ? a.kept + (size_t)unit * a.budget : nullptr;
    if (a.status && unit < a.B * a.Hkv && unit % a.Hkv == 0 && tid == 0) a.status[b] = bad ? S4C_SEQ_BAD_LEN : 0;
    const bool apart = a.weight_out != a.weight, pos_apart = a.key_pos_out != a.key_pos;
    if (bad || n <= a.budget) {
        if (tid == 0) a.meta[unit] = make_int2(0, n);
        if (kept)
            for (int j = tid; j < a.budget; j += kSelect) kept[j] = !bad && j < n ? j : -1;
        if (!bad)
            for (int j = tid; j < n; j += kSelect) {
                if (apart) a.weight_out[row0 + j] = w[j];
                if (pos_apart) a.key_pos_out[row0 + j] = pos[j];
            }
        return;
    }
    const int newest = a.next_pos[b] - a.recent;
    auto key_at = [&](int j) { return key_of(w[j], pos[j] >= newest); };

    // ---- the m-th largest key, from its highest bits down; `left`: how many of the keys with these bits stay
    uint32_t prefix = 0, left = (uint32_t)m;
    int shift = 32;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, lower = shift - bits;
        for (int i = tid; i < kCopies * kBins; i += kSelect) ((uint32_t*)hist)[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kSelect) {
            const uint32_t k = key_at(j);
            if (pass == 0 || (k >> shift) == prefix) atomicAdd(&hist[lane & (kCopies - 1)][(k >> lower) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // thread i has the i-th pair of bins from the top
        const int top = kBins - 1 - 2 * tid;
        uint32_t h0 = 0, h1 = 0;
#pragma unroll
        for (int c = 0; c < kCopies; ++c) { h0 += hist[c][top]; h1 += hist[c][top - 1]; }
        uint32_t incl = h0 + h1;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t y = __shfl_up(incl, off);
            if (lane >= off) incl += y;
        }
        if (lane == 63) s_wave[0][wave] = incl;
        __syncthreads();
        uint32_t before = 0;
        for (int i = 0; i < wave; ++i) before += s_wave[0][i];
        const uint32_t above = before + incl - h0 - h1;              // keys in higher bins
        if (above < left && left <= above + h0) { s_pick[0] = top; s_pick[1] = left - above; }
        else if (above + h0 < left && left <= above + h0 + h1) { s_pick[0] = top - 1; s_pick[1] = left - above - h0; }
        __syncthreads();
        prefix = (prefix << bits) | s_pick[0];
        left = s_pick[1];
        shift = lower;
        __syncthreads();
    }
    const uint32_t least = prefix;                                     // rows of larger keys stay, and the first `left` of this one

    // ---- a wave has a run of rows: how many of them stay before and behind the budget
    const int run = (n + kSelectWaves * 64 - 1) / (kSelectWaves * 64) * 64, j0 = wave * run, j1 = min(n, j0 + run);
    uint32_t more_front = 0, same_front = 0, more_back = 0, same_back = 0;
    for (int j = j0 + lane; j < j1; j += 64) {
        const uint32_t k = key_at(j);
        if (j < m) { more_front += k > least; same_front += k == least; }
        else { more_back += k > least; same_back += k == least; }
    }
    more_front = wave_sum(more_front); same_front = wave_sum(same_front);
    more_back = wave_sum(more_back); same_back = wave_sum(same_back);
    if (lane == 0) { s_wave[0][wave] = more_front; s_wave[1][wave] = same_front; s_wave[2][wave] = more_back; s_wave[3][wave] = same_back; }
    __syncthreads();
    uint32_t same = 0, hole = 0, mover = 0, movers = 0;                // before this wave's rows; of the unit
    {
        uint32_t seen = 0, movers_so_far = 0;
        for (int i = 0; i < kSelectWaves; ++i) {
            if (i == wave) { same = seen; mover = movers_so_far; }
            const uint32_t front = s_wave[1][i], back = s_wave[3][i];
            const uint32_t keep_front = s_wave[0][i] + min(front, left - min(left, seen));
            seen += front;
            const uint32_t keep_back = s_wave[2][i] + min(back, left - min(left, seen));
            seen += back;
            const int f0 = min(m, i * run), f1 = min(m, (i + 1) * run);
            if (i < wave) hole += (uint32_t)(f1 - f0) - keep_front;
            movers_so_far += keep_back;
        }
        movers = movers_so_far;
    }
    if (tid == 0) a.meta[unit] = make_int2((int)movers, m);

    // ---- the lists, in row order
    int32_t* holes = a.lists + (size_t)unit * 2 * a.list_len;
    int32_t* from = holes + a.list_len;
    const unsigned long long below = (1ull << lane) - 1;
    for (int j = j0 + lane; __any(j < j1); j += 64) {
        const bool on = j < j1;
        const uint32_t k = on ? key_at(j) : 0u;
        const unsigned long long eq = __ballot(on && k == least);
        const bool stays = on && (k > least || (k == least && same + __popcll(eq & below) < left));
        same += __popcll(eq);
        const bool is_hole = on && !stays && j < m, moves = stays && j >= m;
        const unsigned long long bh = __ballot(is_hole), bm = __ballot(moves);
        if (is_hole) holes[hole + __popcll(bh & below)] = j;
        if (moves) from[mover + __popcll(bm & below)] = j;
        hole += __popcll(bh);
        mover += __popcll(bm);
        if (stays && j < m) {
            if (kept) kept[j] = j;
            if (apart) a.weight_out[row0 + j] = w[j];
            if (pos_apart) a.key_pos_out[row0 + j] = pos[j];
        }
    }
}

template <int VPR, bool PAGED>       // 16-byte pieces of a row
__global__ __launch_bounds__(kMove) void evict_move_kernel(EvictArgs a) {
    constexpr int kRows = kMove / VPR;
    const int unit = blockIdx.x, ly = unit / (a.B * a.Hkv), b = (unit / a.Hkv) % a.B, h = unit % a.Hkv;
    const int2 meta = a.meta[unit];
    if (blockIdx.y == 0 && threadIdx.x == 0 && unit < a.B * a.Hkv && h == 0) a.new_len[b] = meta.y;
    const int32_t* holes = a.lists + (size_t)unit * 2 * a.list_len;
    const int32_t* from = holes + a.list_len;
    const size_t row0 = (size_t)unit * a.S_cap;
    const int piece = threadIdx.x % VPR;
    const size_t layer = PAGED ? (size_t)ly * a.num_pages * a.Hkv << a.page_shift : 0;
    const int32_t* table = a.block_table + (size_t)b * a.max_blocks;
    auto at = [&](int j) __attribute__((always_inline)) {
        size_t row = row0 + j;
        if constexpr (PAGED) row = layer + (((size_t)table[j >> a.page_shift] * a.Hkv + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        return row * (VPR * 16) + piece * 16;
    };
    for (int i = blockIdx.y * kRows + threadIdx.x / VPR; i < meta.x; i += gridDim.y * kRows) {
        const int src = from[i], dst = holes[i];
        const size_t s = at(src), d = at(dst);
        const u32x4 k = *(const u32x4*)((const char*)a.k_cache + s), v = *(const u32x4*)((const char*)a.v_cache + s);
        if (piece == 0) {
            a.weight_out[row0 + dst] = a.weight[row0 + src];
            a.key_pos_out[row0 + dst] = a.key_pos[row0 + src];
            if (a.kept) a.kept[(size_t)unit * a.budget + dst] = src;
        }
        *(u32x4*)((char*)a.k_cache + d) = k;
        *(u32x4*)((char*)a.v_cache + d) = v;
    }
}

template <int VPR>
void move(const EvictArgs& a, hipStream_t st) {
    const int units = a.layers * a.B * a.Hkv, rows = kMove / VPR;
    int runs = (8 * a.cus + units - 1) / units;
    const int most = (a.list_len + rows - 1) / rows;
    if (runs > most) runs = most < 1 ? 1 : most;
    const dim3 grid((unsigned)units, (unsigned)runs);
    if (a.block_table) hipLaunchKernelGGL((evict_move_kernel<VPR, true>), grid, dim3(kMove), 0, st, a);
    else hipLaunchKernelGGL((evict_move_kernel<VPR, false>), grid, dim3(kMove), 0, st, a);
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)(a.layers * a.B * a.Hkv)), dim3(kSelect), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    switch (a.row_bytes / 16) {
        case 8: move<8>(a, st); break;
        case 16: move<16>(a, st); break;
        default: move<32>(a, st); break;
    }
    return hipGetLastError();
}

}  // namespace s4c
