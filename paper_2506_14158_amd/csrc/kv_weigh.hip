// What the cache rows are worth: the attention weight that the accepted path's query rows give to every cache row, added to the rows'
// totals (s4c_kv_weigh).  weight[j] += sum over path nodes k and the heads of a group of exp(x_kj - lse_k), x as the attention had it.
//
// The log-sum-exp is known, so this is one pass over K: a stream of n D elements per KV head, each feeding 2 R flops (R = path
// nodes x heads of the group).  A wave takes NG x 16 keys: K rows go from memory straight into the B operands of 16x16 matrix
// instructions (a lane has 16 consecutive bytes of a row; the reduction index is permuted the same way for Q), the query rows lie in LDS
// in operand order, and the scores come out with a lane per key, so that a key's sum over the rows is additions in registers and two
// exchanges between the wave's quarters.  No workgroup needs another's result, every sum has one order.
// Measured: 16 x 64/8 heads, 32768 keys, 7 path nodes 214 us (1.1 GB at 5.2 TB/s); 8 x 32/8 heads, 6150 keys on average, paged 23.5 (4.5 TB/s); 32 heads,
// 1029 keys 6, a chain of latencies: lengths, path, query rows.  With many query rows (512 of them, 4096 keys, 16 KV heads: 19.6 us) it is
// bound by what a block of them goes through, LDS, matrix cores, exponentials, and by the start: about 2.7 us for 128 rows and 5 us.  (Multiplying the next block
// while the exponentials of one are taken changed nothing.)
#include <algorithm>

#include "attn_score.h"

namespace s4c {

namespace {

using namespace mfma;
using parts::u32x4;                          // (arrays of HIP's uint4 are not kept in registers)

// Many query rows (below) of 16 bits are shared by eight waves, so that half as many are read and written to LDS: 2 x 8 KV heads, 4096 keys, 512 rows 23.1 and
// 19.6 us; 4 x 8, 20000 keys, 400 rows 133 and 115; 16 x 8, 6000 keys, 168 rows 90 and 79.  Of fp32, with twice the registers a row, by four (8 x 6000
// keys, 400 rows 64 us; 69).
constexpr int waves_of(bool many, size_t element) { return many && element == 2 ? 8 : 4; }
// 16-byte pieces of a row that a lane has: piece 4 t + lane / 16 of its row for t < T.
template <typename E, int D, int NG>
struct Tile {
    static constexpr int kRowB = D * sizeof(E), kT = kRowB / 64, kKeys = 16 * NG;
    static constexpr int kRows = kRowB == 512 ? 64 : 128;        // query rows in LDS at a time
};

template <typename E>
__device__ __forceinline__ f32x4 product(u32x4 q, u32x4 k, f32x4 c) {
    if constexpr (sizeof(E) == 4) {
        const f32x4 x = __builtin_bit_cast(f32x4, q), y = __builtin_bit_cast(f32x4, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
        return c;
    } else {
        return mma16<std::is_same<E, f16_t>::value>(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, k), c);
    }
}

// MANY: the path may have more query rows than lie in LDS at a time.  Then these are replaced while the matrix cores work, chunk by chunk for
// every tile of keys (two buffers, one barrier a chunk).
template <typename E, int D, int NG, bool PAGED, bool MANY>
__global__ __launch_bounds__(64 * waves_of(MANY, sizeof(E)), 2) void kv_weigh_kernel(WeighArgs a) {
    constexpr int kWaves = waves_of(MANY, sizeof(E)), kThreads = 64 * kWaves;
    typedef Tile<E, D, NG> T;
    constexpr int kBufs = MANY ? 2 : 1, kTogether = MANY && NG < 4 ? 2 : 1;      // blocks of 16 rows at a time
    __shared__ __attribute__((aligned(16))) unsigned char s_q[kBufs][T::kRows * T::kRowB];     // [16-row block][piece t][lane] 16 bytes
    __shared__ __attribute__((aligned(16))) float s_lse[kBufs][T::kRows], s_slope[kBufs][T::kRows];
    __shared__ int s_node[kBufs][T::kRows];
    __shared__ int s_path[kMaxNodes];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int unit = blockIdx.x, b = unit / a.Hkv, kvh = unit - b * a.Hkv;
    const int n = a.cache_len[b], L = a.accept_len[b];
    const int32_t* path = a.path + (size_t)b * a.max_path;

    const bool off_limits = n < 1 || n > a.max_cache_len || n > a.S_cap || L < 0 || L >= a.max_path || L + 1 > n;
    if (off_limits) {
        if (a.status && blockIdx.y == 0 && kvh == 0 && tid == 0) a.status[b] = S4C_SEQ_BAD_LEN;
        return;
    }
    const int first = n - (L + 1), R = (L + 1) * a.G, chunks = MANY ? (R + T::kRows - 1) / T::kRows : 1;
    // this workgroup's keys, in steps of all its waves' tiles
    constexpr int kStep = kWaves * T::kKeys;
    const int steps = (n + kStep - 1) / kStep, per = (steps + (int)gridDim.y - 1) / (int)gridDim.y;
    const int step0 = blockIdx.y * per, step1 = min(steps, step0 + per);
    if (step0 >= step1) return;
    // (nodes are used before the path has been looked over)
    auto node_of = [&](int node) __attribute__((always_inline)) { return min(max(node, 0), a.N - 1); };
    if constexpr (MANY)
        if (tid < kMaxNodes) s_path[tid] = tid <= L ? path[tid] : 0;

    // Query rows c kRows ..: into registers (nothing is done with them there that would wait for them), and from there into a buffer.  A thread
    // has every kThreads-th 16-byte place of the buffer, so that a wave writes a kilobyte in a row: lane r + 16 p of 64 places has piece
    // 4 t + p of row r of a block (with a thread's pieces in one row each, 16 lanes wrote to the same banks, 1 us a chunk).
    constexpr int kMine = T::kRows * T::kRowB / 16 / kThreads, kBlocksApart = kThreads / 64 >= T::kT ? kThreads / 64 / T::kT : 1;
    const int my_row = ((tid >> 6) / T::kT) * 16 + (tid & 15);
    auto my_piece = [&](int i) __attribute__((always_inline)) { return 4 * (((tid >> 6) + i * (kThreads / 64)) % T::kT) + ((tid >> 4) & 3); };
    auto same_row = [](int i) { return (i * (kThreads / 64)) % T::kT != 0; };                 // as place i - 1
    const int step_k = 16 * kBlocksApart / a.G, step_g = 16 * kBlocksApart - step_k * a.G;
    const unsigned char* const q0 = (const unsigned char*)a.q + ((size_t)b * a.N * a.Hq + kvh * a.G) * T::kRowB;
    auto rows_of = [&](int c) __attribute__((always_inline)) { return (min(T::kRows, R - c * T::kRows) + 16 * kTogether - 1) / (16 * kTogether) * (16 * kTogether); };
    u32x4 row[kMine];
    float row_lse = INFINITY, row_slope = 0.f;
    int row_k = 0;
    auto load = [&](int c, auto in_lds) __attribute__((always_inline)) {
        auto node_at = [&](int k) __attribute__((always_inline)) { return node_of(decltype(in_lds)::value ? s_path[k] : path[k]); };
        const int r0 = c * T::kRows;
        int k = (r0 + my_row) / a.G, g = r0 + my_row - k * a.G;
        int node[kMine], head[kMine];
        row_k = (r0 + tid) / a.G;
        const int row_g = r0 + tid - row_k * a.G;
        const bool row_on = tid < T::kRows && r0 + tid < R;
        const int row_node = node_at(row_on ? row_k : 0);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {                              // (behind the last row: that one again)
            if (same_row(i)) {
                node[i] = node[i - 1];
                head[i] = head[i - 1];
                continue;
            }
            if (i > 0) {
                k += step_k;
                g += step_g;
                if (g >= a.G) { g -= a.G; ++k; }
            }
            node[i] = node_at(min(k, L));
            head[i] = k > L ? a.G - 1 : g;
        }
#pragma unroll
        for (int i = 0; i < kMine; ++i) row[i] = *(const u32x4*)(q0 + ((size_t)node[i] * a.Hq + head[i]) * T::kRowB + 16 * my_piece(i));
        row_lse = INFINITY;                                            // rows that do not exist give no weight
        if (row_on) {
            row_lse = a.lse[((size_t)b * a.N + row_node) * a.Hq + kvh * a.G + row_g];
            if (a.score.slopes) row_slope = a.score.slopes[kvh * a.G + row_g];
        }
    };
    auto store = [&](int buf, int c) __attribute__((always_inline)) {
        const int up = rows_of(c);
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (((i * (kThreads / 64)) / T::kT) * 16 < up) *(u32x4*)(s_q[buf] + (tid + i * kThreads) * 16) = row[i];
        if (tid < T::kRows) { s_lse[buf][tid] = row_lse * kLog2e; s_slope[buf][tid] = row_slope * kLog2e; s_node[buf][tid] = row_k; }
    };

    const int root = a.score.key_pos ? a.score.root_pos[b] : first;
    const size_t row0 = ((size_t)b * a.Hkv + kvh) * a.S_cap;           // of the totals and positions
    u32x4 kf[NG][T::kT], nf[NG][T::kT];
    int pos[NG], npos[NG];
    float total, ntotal;
    auto fetch = [&](int step, u32x4 (&f)[NG][T::kT], int (&p)[NG], float& w) __attribute__((always_inline)) {
        const int j0 = __builtin_amdgcn_readfirstlane(step * kStep + wave * T::kKeys);
        size_t row = row0 + j0;
        if constexpr (PAGED) {
            const int jc = min(j0, n - 1) & ~(T::kKeys - 1);
            int id = a.block_table[(size_t)b * a.max_blocks + (jc >> a.page_shift)];
            id = (unsigned)id < (unsigned)a.num_pages ? id : 0;
            row = (((size_t)id * a.Hkv + kvh) << a.page_shift) + (jc & ((1 << a.page_shift) - 1));
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int in = 16 * g + (lane & 15);
            const int j = min(j0 + in, n - 1);
            // (a tile behind the last key: the last one's rows; never multiplied into anything that is kept)
            const int off = PAGED ? j - (min(j0, n - 1) & ~(T::kKeys - 1)) : j - j0;
            const unsigned char* src = (const unsigned char*)a.k_cache + (ptrdiff_t)(row + (ptrdiff_t)off) * T::kRowB + (lane >> 4) * 16;
#pragma unroll
            for (int t = 0; t < T::kT; ++t) f[g][t] = *(const u32x4*)(src + 64 * t);
            p[g] = a.score.slopes && a.score.key_pos ? a.score.key_pos[row0 + j] : j;
        }
        w = a.weight_in[row0 + min(j0 + (lane & (T::kKeys - 1)), n - 1)];
    };

    // The keys, the query rows and what tells whether they are the sequence's are requested together; every address is in bounds
    // whatever the path and the table hold.
    fetch(step0, nf, npos, ntotal);
    bool bad = false;
    for (int k = tid; k <= L; k += kThreads) bad = bad || path[k] < 0 || path[k] >= a.N;
    if constexpr (PAGED)
        for (int i = tid; i < (n + (1 << a.page_shift) - 1) >> a.page_shift; i += kThreads) {
            const int id = a.block_table[(size_t)b * a.max_blocks + i];
            bad = bad || id < 0 || id >= a.num_pages;
        }
    load(0, std::false_type());
    store(0, 0);
    bad = __syncthreads_or(bad) != 0;                                  // (every workgroup finds the same)
    if (a.status && blockIdx.y == 0 && kvh == 0 && tid == 0) a.status[b] = bad ? S4C_SEQ_BAD_LEN : 0;
    if (bad) return;
    int buf = 0;
    for (int step = step0; step < step1; ++step) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int t = 0; t < T::kT; ++t) kf[g][t] = nf[g][t];
            pos[g] = npos[g];
        }
        total = ntotal;
        if (step + 1 < step1) fetch(step + 1, nf, npos, ntotal);
        const int j0 = step * kStep + wave * T::kKeys;
        const bool own_rows = j0 + T::kKeys > first;                   // some keys are the path's own
        float rel[NG], sum[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int j = j0 + 16 * g + (lane & 15);
            rel[g] = (float)(j >= first ? j - first : pos[g] - root);
            sum[g] = 0.f;
        }
        for (int c = 0; c < chunks; ++c) {
            const bool more = MANY && chunks > 1 && (c + 1 < chunks || step + 1 < step1);
            // (a choice for every row would wait for the rows before it)
            if (more && L < kMaxNodes) load(c + 1 < chunks ? c + 1 : 0, std::true_type());
            else if (more) load(c + 1 < chunks ? c + 1 : 0, std::false_type());
            const int blocks = rows_of(c) / 16;
            for (int blk = 0; blk < blocks; blk += kTogether) {
                f32x4 s[kTogether * NG];
#pragma unroll
                for (int i = 0; i < kTogether * NG; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                u32x4 q[kTogether][T::kT];
#pragma unroll
                for (int u = 0; u < kTogether; ++u)
#pragma unroll
                    for (int t = 0; t < T::kT; ++t) q[u][t] = *(const u32x4*)(s_q[buf] + (((blk + u) * T::kT + t) * 64 + lane) * 16);
                f32x4 lse[kTogether], slope[kTogether];
#pragma unroll
                for (int u = 0; u < kTogether; ++u) {
                    lse[u] = *(const f32x4*)(s_lse[buf] + (blk + u) * 16 + 4 * (lane >> 4));
                    if (a.score.slopes) slope[u] = *(const f32x4*)(s_slope[buf] + (blk + u) * 16 + 4 * (lane >> 4));
                }
#pragma unroll
                for (int t = 0; t < T::kT; ++t)
#pragma unroll
                    for (int u = 0; u < kTogether; ++u)
#pragma unroll
                        for (int g = 0; g < NG; ++g) s[u * NG + g] = product<E>(q[u][t], kf[g][t], s[u * NG + g]);
                if (a.score.cap_log2 > 0.f) score::cap(s, a.score, a.score.cap_log2);
                if (own_rows) {
#pragma unroll
                    for (int u = 0; u < kTogether; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int last = first + s_node[buf][(blk + u) * 16 + 4 * (lane >> 4) + e];
#pragma unroll
                            for (int g = 0; g < NG; ++g)
                                if (j0 + 16 * g + (lane & 15) > last) s[u * NG + g][e] = -INFINITY;
                        }
                }
                if (a.score.slopes) {
#pragma unroll
                    for (int u = 0; u < kTogether; ++u)
#pragma unroll
                        for (int g = 0; g < NG; ++g)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[g] += fast_exp2(fmaf(s[u * NG + g][e], a.score.mul, fmaf(slope[u][e], rel[g], -lse[u][e])));
                } else {
#pragma unroll
                    for (int u = 0; u < kTogether; ++u)
#pragma unroll
                        for (int g = 0; g < NG; ++g)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[g] += fast_exp2(fmaf(s[u * NG + g][e], a.score.mul, -lse[u][e]));
                }
            }
            if (more) {                                                // (what the other buffer held was read before the last barrier)
                store(buf ^ 1, c + 1 < chunks ? c + 1 : 0);
                __syncthreads();
                buf ^= 1;
            }
        }
        // lane 16 g + i has key 16 g + i of the tile
        float mine = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            sum[g] += __shfl_xor(sum[g], 16);
            sum[g] += __shfl_xor(sum[g], 32);
            if ((lane >> 4) == g) mine = sum[g];
        }
        const int j = j0 + lane;
        if (lane < T::kKeys && j < n) {
            a.weight[row0 + j] = j < first ? total + mine : mine;
            if (a.score.key_pos && j >= first) a.key_pos[row0 + j] = root + (j - first);
        }
    }
}

template <typename E, int D, int NG, bool MANY>
hipError_t launch(const WeighArgs& a, int runs, hipStream_t st) {
    const dim3 grid((unsigned)(a.B * a.Hkv), (unsigned)runs), block(64 * waves_of(MANY, sizeof(E)));
    if (a.block_table) hipLaunchKernelGGL((kv_weigh_kernel<E, D, NG, true, MANY>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv_weigh_kernel<E, D, NG, false, MANY>), grid, block, 0, st, a);
    return hipGetLastError();
}
// Few query rows: tiles of half as many keys, four workgroups for a CU (three of which run at a time), unless there are many keys: then whole tiles,
// two workgroups on a CU, each with a longer run (bf16, head size 128, units x keys, whole and half tiles, us: 32 x 1029 7.7 and 6.3; 160 x 1000 13.7 and
// 11.2; 128 x 2000 17.9 and 16.3; 128 x 8000 58.4 and 56.7; 128 x 32768 208 and 216).
// Many, 16 bits: whole tiles, which read the query rows from LDS half as often, where they fill the chip (units x keys, rows, whole and half, us: 8 x 8192,
// 512 29.4 and 19.8; 8 x 16384, 512 31.3 and 33.3; 16 x 16384, 512 54.2 and 58.8; 128 x 2000, 168 28.8 and 31.6; 128 x 6000, 168 70 and 79; 32 x 20000,
// 400 100 and 110).  One workgroup of eight waves runs on a CU at a time.
// Where workgroups run long, one more than run at a time takes as long as twice as many: runs are chosen by the turns they take (units x keys, rows, workgroups,
// us: 24 x 16384, 512: 264 124, 240 92; 320 x 4000, 168: 320 206, 640 146; whole tiles of few rows: 72 x 16000: 576 71, 504 61; 160 x 16000: 640 142,
// 480 133; 520 x 3000: 520 105, 1560 91).
template <typename E, int D, int NG>
hipError_t launch_tiles(const WeighArgs& a, hipStream_t st) {
    const long long units = (long long)a.B * a.Hkv;
    auto steps = [&](long long step) { return (a.max_cache_len + step - 1) / step; };
    auto runs = [&](int per_cu, long long n) { return (int)std::min((per_cu * a.cus + units - 1) / units, n); };
    auto shared_out = [&](long long at_once, long long n) {           // n steps a unit -> runs; the start of a run takes as long as a step
        const long long least_turns = (units + at_once - 1) / at_once;
        long long best = 1, least = 0;
        for (long long turns = least_turns; turns < least_turns + 4; ++turns) {
            const long long most = std::min(turns * at_once / units, n), cost = turns * ((n + most - 1) / most + 1);
            if (least == 0 || cost < least) { least = cost; best = most; }
        }
        return (int)best;
    };
    if ((long long)a.max_path * a.G > Tile<E, D, NG>::kRows) {
        constexpr int kWaves = waves_of(true, sizeof(E));
        const long long whole = steps(kWaves * 16 * NG), half = steps(kWaves * 8 * NG);
        if constexpr (kWaves == 8)
            return units * whole >= a.cus ? launch<E, D, NG, true>(a, shared_out(a.cus, whole), st) : launch<E, D, NG / 2, true>(a, shared_out(a.cus, half), st);
        else
            return launch<E, D, NG / 2, true>(a, runs(4, half), st);
    }
    constexpr int kWaves = waves_of(false, sizeof(E));
    const long long whole = steps(kWaves * 16 * NG);
    if (units * whole <= 16ll * a.cus) return launch<E, D, NG / 2, false>(a, runs(4, steps(kWaves * 8 * NG)), st);
    return launch<E, D, NG, false>(a, shared_out(2 * a.cus, whole), st);
}

}  // namespace

hipError_t launch_weigh(const WeighArgs& a, int dtype, hipStream_t st) {
    if (dtype == S4C_F32) return a.D == 64 ? launch_tiles<float, 64, 4>(a, st) : launch_tiles<float, 128, 2>(a, st);
    if (dtype == S4C_F16) return a.D == 64 ? launch_tiles<f16_t, 64, 4>(a, st) : launch_tiles<f16_t, 128, 4>(a, st);
    return a.D == 64 ? launch_tiles<bf16_t, 64, 4>(a, st) : launch_tiles<bf16_t, 128, 4>(a, st);
}

}  // namespace s4c
