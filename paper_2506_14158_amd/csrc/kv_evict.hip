// A cache cut down to a budget (s4c_kv_evict): of every (layer, sequence, KV head) the most recent rows stay, and of the others those
// with the largest totals of attention weight (equal ones: lowest row first), `budget` rows altogether.
//
// Rows that stay and lie behind the budget move into the places that evicted rows leave before it, the i-th into the i-th: every source
// lies behind the budget and every place before it, so rows move in any order, in place, and no more of them than must.  (Attention does
// not ask for an order of the keys; what depends on a row's age reads its position.)
//
// Selection, a workgroup per unit.  A row's key is its total's bits in integer order, all ones if it is recent; the keys of up to 32768 rows
// are kept in LDS (longer units are read again for every sweep).  The smallest key that stays is found by a radix descent, 11, 11
// and 10 bits from the top: a histogram in LDS, which every wave scans by itself (a barrier less, and nothing to hand over), and the last digits are
// left out where all rows of a bin stay, as they do as soon as totals differ.  Places and movers are listed in row order by ballots.  What bounds it is
// the instructions of one CU on a long unit: 128 units of up to 32768 rows 28 us (keys read from memory in every sweep 94, more instructions a key 54).
// Moving is a copy, bound by memory: 9500 rows of 256 bytes of each of them, K and V, 167 us (833 MB, 5.0 TB/s).
// 32 layers of 32 heads, 1367 -> 1024 rows, in one launch 79 us, 355 MB at 4.5 TB/s.
#include "mfma_common.h"

namespace s4c {

namespace {

constexpr int kBins = 2048;
constexpr int kMostKeys = 32768;             // in LDS
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A total's bits in the order of the numbers, 2^21 .. 2^32 - 2 (-0 as 0); recent rows: 2^32 - 1.  So the first digit of a key is never 0, nor is the smallest
// that stays, whatever the totals hold: 0 stands for rows that do not exist.
__device__ __forceinline__ uint32_t key_of(float w, bool recent) {
    const uint32_t u = __float_as_uint(w + 0.f);
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return recent ? 0xFFFFFFFFu : min(max(k, 1u << 21), 0xFFFFFFFEu);
}

// Where bin d of a histogram lies: a scanning lane l reads bins 32 l .. 32 l + 31, each time all lanes from different banks.
__device__ __forceinline__ uint32_t bin_at(uint32_t d) { return d ^ (d >> 5); }

__device__ __forceinline__ uint32_t wave_inclusive(uint32_t x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    return x;
}

// One more in bin d for every lane that is `on`.  Lanes that add to one word wait for each other; CROWDED, where most keys may share a bin, one lane
// adds for all if all agree.
template <bool CROWDED>
__device__ __forceinline__ void count(uint32_t* hist, bool on, uint32_t d) {
    if constexpr (CROWDED) {
        const unsigned long long who = __ballot(on);
        if (who == 0) return;
        const int one = __ffsll((long long)who) - 1;
        if (__ballot(on && d == __builtin_amdgcn_readlane(d, one)) == who) {
            if ((int)(threadIdx.x & 63) == one) atomicAdd(&hist[bin_at(d)], (uint32_t)__popcll(who));
            return;
        }
    }
    if (on) atomicAdd(&hist[bin_at(d)], 1u);
}

// n words from `from` to `to`, by the threads of a workgroup
template <int THREADS>
__device__ __forceinline__ void copy_words(uint32_t* to, const uint32_t* from, int n) {
    if (((((uintptr_t)to) | ((uintptr_t)from)) & 15) == 0) {
        for (int i = threadIdx.x; i < n / 4; i += THREADS) ((u32x4*)to)[i] = ((const u32x4*)from)[i];
        const int i = n / 4 * 4 + threadIdx.x;
        if (i < n) to[i] = from[i];
    } else {
        for (int i = threadIdx.x; i < n; i += THREADS) to[i] = from[i];
    }
}

// Rows i, i + step, .. of a unit's list move, by the threads of a workgroup: VPR 16-byte pieces of a row, K and V.  Every byte is touched once, and
// passes the caches by (128 units of 16384 rows of 256 bytes, 9500 of which move: 183 us and 165).
template <int VPR, bool PAGED>
__device__ __forceinline__ void move_rows(const EvictArgs& a, int unit, int threads, int count, int part, int parts) {
    constexpr int kBatch = 4;                // rows in flight
    const int ly = unit / (a.B * a.Hkv), b = (unit / a.Hkv) % a.B, h = unit % a.Hkv;
    const int32_t* holes = a.lists + (size_t)unit * 2 * a.list_len;
    const int32_t* from = holes + a.list_len;
    const size_t row0 = (size_t)unit * a.S_cap;
    const int piece = threadIdx.x % VPR, rows = threads / VPR;
    const size_t layer = PAGED ? (size_t)ly * a.num_pages * a.Hkv << a.page_shift : 0;
    const int32_t* table = a.block_table + (size_t)b * a.max_blocks;
    auto at = [&](int j) __attribute__((always_inline)) {
        size_t row = row0 + j;
        if constexpr (PAGED) row = layer + (((size_t)table[j >> a.page_shift] * a.Hkv + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        return row * (VPR * 16) + piece * 16;
    };
    for (int i0 = part * rows * kBatch + threadIdx.x / VPR; i0 < count; i0 += parts * rows * kBatch) {
        int src[kBatch], dst[kBatch];
        size_t s[kBatch], d[kBatch];
        u32x4 k[kBatch], v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = min(i0 + u * rows, count - 1);
            src[u] = from[i];
            dst[u] = holes[i];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            s[u] = at(src[u]);
            d[u] = at(dst[u]);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            k[u] = __builtin_nontemporal_load((const u32x4*)((const char*)a.k_cache + s[u]));
            v[u] = __builtin_nontemporal_load((const u32x4*)((const char*)a.v_cache + s[u]));
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u * rows >= count) continue;
            if (piece == u) {                // (a lane of the row each, so that the batch's reads go out together)
                a.weight_out[row0 + dst[u]] = a.weight[row0 + src[u]];
                a.key_pos_out[row0 + dst[u]] = a.key_pos[row0 + src[u]];
                if (a.kept) a.kept[(size_t)unit * a.budget + dst[u]] = src[u];
            }
            __builtin_nontemporal_store(k[u], (u32x4*)((char*)a.k_cache + d[u]));
            __builtin_nontemporal_store(v[u], (u32x4*)((char*)a.v_cache + d[u]));
        }
    }
}

// VPR > 0: the workgroup moves its unit's rows too, and new_len is written here unless it is cache_len, which others may not have read.
// Otherwise a second one for every unit (blockIdx.y) writes what lies before the budget as it is; movers come over it.
template <int WAVES, int VPR, bool PAGED>
__global__ __launch_bounds__(WAVES * 64) void evict_select_kernel(EvictArgs a) {
    constexpr int kThreads = WAVES * 64;
    __shared__ uint32_t hist[3][kBins];
    __shared__ uint32_t s_count[WAVES][4];
    __shared__ uint32_t s_recent[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int unit = blockIdx.x, b = (unit / a.Hkv) % a.B;
    const int n = a.cache_len[b];
    bool bad = n < 0 || n > a.S_cap;
    if constexpr (PAGED)
        if (!bad)
            for (int i = tid; i < (n + (1 << a.page_shift) - 1) >> a.page_shift; i += kThreads) {
                const int id = a.block_table[(size_t)b * a.max_blocks + i];
                bad = bad || id < 0 || id >= a.num_pages;
            }
    for (int i = tid; i < 3 * kBins; i += kThreads) ((uint32_t*)hist)[i] = 0;
    bad = __syncthreads_or(bad) != 0;
    const int m = min(n, a.budget);
    const size_t row0 = (size_t)unit * a.S_cap;
    const float* w = a.weight + row0;
    const int32_t* pos = a.key_pos + row0;
    int32_t* kept = a.kept ? a.kept + (size_t)unit * a.budget : nullptr;
    if (unit < a.B * a.Hkv && unit % a.Hkv == 0 && tid == 0 && blockIdx.y == 0) {
        if (a.status) a.status[b] = bad ? S4C_SEQ_BAD_LEN : 0;
        if (VPR > 0 && a.new_len != a.cache_len) a.new_len[b] = bad ? n : m;
    }
    const bool apart = a.weight_out != a.weight, pos_apart = a.key_pos_out != a.key_pos;
    auto write_front = [&]() __attribute__((always_inline)) {
        if (apart) copy_words<kThreads>((uint32_t*)a.weight_out + row0, (const uint32_t*)w, m);
        if (pos_apart) copy_words<kThreads>((uint32_t*)a.key_pos_out + row0, (const uint32_t*)pos, m);
        if (kept)
            for (int j = tid; j < m; j += kThreads) kept[j] = j;
    };
    if (VPR == 0 && blockIdx.y > 0) {
        if (!bad && n > a.budget) write_front();
        return;
    }
    if (bad || n <= a.budget) {
        if (tid == 0) a.meta[unit] = make_int2(0, n);
        if (kept)
            for (int j = tid; j < a.budget; j += kThreads) kept[j] = !bad && j < n ? j : -1;
        if (!bad)
            for (int j = tid; j < n; j += kThreads) {
                if (apart) a.weight_out[row0 + j] = w[j];
                if (pos_apart) a.key_pos_out[row0 + j] = pos[j];
            }
        return;
    }
    const int newest = a.next_pos[b] - a.recent;

    // ---- keys: a wave has a run of rows, 64 at a time
    extern __shared__ uint32_t keys[];
    const bool here = n <= a.lds_keys;
    const int run = (n + kThreads - 1) / kThreads * 64, j0 = wave * run, j1 = min(n, j0 + run);
    // f(j, key): of this wave's rows j .. j + 63, each lane its own; 0 for a row that does not exist.  Four reads go out together.
    auto every = [&](auto f) __attribute__((always_inline)) {
        auto walk = [&](auto get) __attribute__((always_inline)) {
            for (int jw = j0; jw < j1; jw += 256) {
                uint32_t k[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) k[i] = get(min(jw + 64 * i + lane, n - 1));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (jw + 64 * i < j1) f(jw + 64 * i, jw + 64 * i + lane < j1 ? k[i] : 0u);
            }
        };
        if (here) walk([&](int j) __attribute__((always_inline)) { return keys[j]; });
        else walk([&](int j) __attribute__((always_inline)) { return key_of(w[j], pos[j] >= newest); });
    };
    // The first look.  Every load of a turn is in flight at once.
    constexpr int kLook = WAVES == 16 ? 16 : 8;
    uint32_t recents = 0;
    for (int jw = j0; jw < j1; jw += 64 * kLook) {
        float x[kLook];
        int p[kLook];
#pragma unroll
        for (int i = 0; i < kLook; ++i) {
            const int j = min(jw + 64 * i + lane, n - 1);
            x[i] = w[j];
            p[i] = pos[j];
        }
#pragma unroll
        for (int i = 0; i < kLook; ++i) {
            const int j = jw + 64 * i + lane;
            const bool on = j < j1, recent = p[i] >= newest;
            const uint32_t k = key_of(x[i], recent);
            recents += __popcll(__ballot(on && recent));
            count<false>(hist[0], on && !recent, ~k >> 21);
            if (on && here) keys[j] = k;
        }
    }
    if (lane == 0) s_recent[wave] = recents;
    if constexpr (VPR > 0) write_front();
    __syncthreads();

    // ---- the m-th largest key, from its highest bits down; recent rows, which come first, were counted by themselves
    uint32_t prefix = 0, left = (uint32_t)m;           // of the keys with these bits, `left` stay
    uint32_t least = 0xFFFFFFFFu;                      // rows of larger keys stay, and the first `left` of this one
    recents = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) recents += s_recent[i];
    const bool others = recents < (uint32_t)m;         // some of them stay
    if (others) left -= recents;
    uint32_t in = 0;                                   // keys of the bin
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        if (!others) break;
        const int bits = pass < 2 ? 11 : 10, lower = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        if (pass > 0) {
            auto look = [&](auto crowded) __attribute__((always_inline)) {
                every([&](int, uint32_t k) __attribute__((always_inline)) {
                    count<decltype(crowded)::value>(hist[pass], k != 0xFFFFFFFFu && k >> ((lower + bits) & 31) == prefix && k != 0,
                                                    (~k >> lower) & ((1u << bits) - 1u));
                });
            };
            if (in * 8 > (uint32_t)n) look(std::integral_constant<bool, true>{});
            else look(std::integral_constant<bool, false>{});
            __syncthreads();
        }
        // lane l has bins 32 l .. of the digit's complement, larger keys first: which lane's, then which of them
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) sum += hist[pass][bin_at(32 * lane + i)];
        uint32_t incl = wave_inclusive(sum);
        const int at = __ffsll((long long)__ballot(incl >= left)) - 1;
        left -= __builtin_amdgcn_readlane(incl - sum, at);
        sum = lane < 32 ? hist[pass][bin_at(32 * at + lane)] : 0u;
        incl = wave_inclusive(sum);
        const int bin = __ffsll((long long)__ballot(incl >= left)) - 1;
        left -= __builtin_amdgcn_readlane(incl - sum, bin);
        in = __builtin_amdgcn_readlane(sum, bin);
        const uint32_t digit = (uint32_t)(32 * at + bin);
        prefix = (prefix << bits) | (~digit & ((1u << bits) - 1u));
        least = prefix << lower;
        if (in == left) {                              // all of the bin
            left = 0xFFFFFFFFu;
            break;
        }
    }

    // ---- the lists, in row order.  `left` equal rows stay; all of them where nothing was left over
    int32_t* holes = a.lists + (size_t)unit * 2 * a.list_len;
    int32_t* from = holes + a.list_len;
    const unsigned long long below = (1ull << lane) - 1;
    const bool tied = left != 0xFFFFFFFFu;
    uint32_t same = 0, hole = 0, mover = 0, movers = 0;                // before this wave's rows; of the unit
    if (here) {
        // A wave lists its rows over the keys it has read, places first (rows before the budget come first); where its lists begin is known
        // when all waves have theirs.
        if (tied) {
            uint32_t eq = 0;
            every([&](int, uint32_t k) __attribute__((always_inline)) { eq += __popcll(__ballot(k == least)); });
            if (lane == 0) s_count[wave][2] = eq;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) same += i < wave ? s_count[i][2] : 0u;
        }
        uint32_t mine = 0, my_holes = 0;
        auto note = [&](unsigned long long who, int jw) __attribute__((always_inline)) {
            if ((who >> lane) & 1) keys[j0 + mine + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = jw + lane;
            mine += __popcll(who);
        };
        auto stays = [&](uint32_t k) __attribute__((always_inline)) {
            if (!tied) return __ballot(k >= least);
            const unsigned long long eq = __ballot(k == least);
            const bool s = k > least || (k == least && same + __popcll(eq & below) < left);
            same += __popcll(eq);
            return __ballot(s);
        };
        // (four blocks are read before the first of them is written over)
        int jw = j0;
        const int front_end = min(j1, m);
        for (; jw + 256 <= front_end; jw += 256) {
            uint32_t k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = keys[jw + 64 * i + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) note(~stays(k[i]), jw + 64 * i);
        }
        for (; jw + 64 <= front_end; jw += 64) note(~stays(keys[jw + lane]), jw);
        if (jw < front_end) {                          // the rows on both sides of the budget
            const unsigned long long st = stays(jw + lane < j1 ? keys[jw + lane] : 0u), front = (1ull << (m - jw)) - 1;
            note(~st & front, jw);
            my_holes = mine;
            note(st & ~front, jw);
            jw += 64;
        } else {
            my_holes = mine;
        }
        for (; jw + 256 <= j1; jw += 256) {
            uint32_t k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = keys[jw + 64 * i + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) note(stays(k[i]), jw + 64 * i);
        }
        for (; jw < j1; jw += 64) note(stays(jw + lane < j1 ? keys[jw + lane] : 0u), jw);
        if (lane == 0) { s_count[wave][0] = my_holes; s_count[wave][1] = mine - my_holes; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            if (i == wave) mover = movers;
            if (i < wave) hole += s_count[i][0];
            movers += s_count[i][1];
        }
        for (uint32_t i = lane; i < my_holes; i += 64) holes[hole + i] = keys[j0 + i];
        for (uint32_t i = lane; i < mine - my_holes; i += 64) from[mover + i] = keys[j0 + my_holes + i];
    } else {
        // Longer units: counted first, then listed in place.
        uint32_t more_front = 0, same_front = 0, more_back = 0, same_back = 0;
        every([&](int jw, uint32_t k) __attribute__((always_inline)) {
            const unsigned long long gt = __ballot(k > least), eq = __ballot(k == least), front = m - jw >= 64 ? ~0ull : m > jw ? (1ull << (m - jw)) - 1 : 0ull;
            more_front += __popcll(gt & front); same_front += __popcll(eq & front);
            more_back += __popcll(gt & ~front); same_back += __popcll(eq & ~front);
        });
        if (lane == 0) { s_count[wave][0] = more_front; s_count[wave][1] = same_front; s_count[wave][2] = more_back; s_count[wave][3] = same_back; }
        __syncthreads();
        uint32_t seen = 0;
        for (int i = 0; i < WAVES; ++i) {
            if (i == wave) { same = seen; mover = movers; }
            const uint32_t keep_front = s_count[i][0] + min(s_count[i][1], left - min(left, seen));
            seen += s_count[i][1];
            const uint32_t keep_back = s_count[i][2] + min(s_count[i][3], left - min(left, seen));
            seen += s_count[i][3];
            if (i < wave) hole += (uint32_t)(min(m, (i + 1) * run) - min(m, i * run)) - keep_front;
            movers += keep_back;
        }
        every([&](int jw, uint32_t k) __attribute__((always_inline)) {
            const int j = jw + lane;
            const unsigned long long eq = __ballot(k == least);
            const bool stays = k > least || (k == least && same + __popcll(eq & below) < left);
            same += __popcll(eq);
            const bool is_hole = k != 0 && j < m && !stays, moves = j >= m && stays;
            const unsigned long long bh = __ballot(is_hole), bm = __ballot(moves);
            if (is_hole) holes[hole + __popcll(bh & below)] = j;
            if (moves) from[mover + __popcll(bm & below)] = j;
            hole += __popcll(bh);
            mover += __popcll(bm);
        });
    }
    if (tid == 0) a.meta[unit] = make_int2((int)movers, m);
    if constexpr (VPR > 0) {
        __syncthreads();
        move_rows<VPR, PAGED>(a, unit, kThreads, (int)movers, 0, 1);
    }
}

constexpr int kMove = 256;

template <int VPR, bool PAGED>
__global__ __launch_bounds__(kMove) void evict_move_kernel(EvictArgs a) {
    const int unit = blockIdx.x;
    const int2 meta = a.meta[unit];
    if (blockIdx.y == 0 && threadIdx.x == 0 && unit < a.B * a.Hkv && unit % a.Hkv == 0) a.new_len[(unit / a.Hkv) % a.B] = meta.y;
    move_rows<VPR, PAGED>(a, unit, kMove, meta.x, blockIdx.y, gridDim.y);
}

// the lengths alone, where every workgroup has moved its unit's rows
__global__ void evict_lengths_kernel(EvictArgs a) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < a.B) a.new_len[b] = a.meta[b * a.Hkv].y;
}

template <int WAVES, int VPR, bool PAGED>
hipError_t select(EvictArgs a, int keys, hipStream_t st) {
    static std::atomic<uint64_t> lds_set{0};
    constexpr int kMost = (WAVES == 4 ? 8192 : kMostKeys) * 4;
    const hipError_t e = ensure_dynamic_lds((const void*)evict_select_kernel<WAVES, VPR, PAGED>, kMost, lds_set);
    if (e != hipSuccess) return e;
    a.lds_keys = keys;
    const bool front = VPR == 0 && (a.kept || a.weight_out != a.weight || a.key_pos_out != a.key_pos);
    const dim3 grid((unsigned)(a.layers * a.B * a.Hkv), front ? 2u : 1u);
    hipLaunchKernelGGL((evict_select_kernel<WAVES, VPR, PAGED>), grid, dim3(WAVES * 64), keys * 4, st, a);
    return hipGetLastError();
}

template <int VPR, bool PAGED>
hipError_t launch(const EvictArgs& a, hipStream_t st) {
    const int units = a.layers * a.B * a.Hkv;
    const int keys = a.S_cap < kMostKeys ? a.S_cap : kMostKeys;
    // Who selects moves as well, in four waves, where there are units enough to fill the chip (others are selected meanwhile), or next to nothing to move.
    // One launch and two, us (units x rows -> budget, bf16, head size 128): 512 x 1000 -> 700 39.7 and 41.6, 1024 x 4000 -> 2000 290 and 304, 512 x 8000 ->
    // 4000 292 and 307, but 256 x 4000 -> 2000 88 and 82, 64 x 8000 -> 4000 127 and 56; 128 x 300 -> 200 9.6 and 17.2, but 8 x 1000 -> 700 12.2 and 10.3.
    const bool whole = a.S_cap <= 8192 && (units >= 2 * a.cus || (a.S_cap <= 2048 && (long long)a.list_len * a.row_bytes <= 65536));
    // (selection alone, four waves and sixteen: 128 x 2000 22.2 and 24.8, 128 x 4000 48.7 and 48.3, 128 x 8000 88.8 and 82.9 with the moving)
    const bool few = a.S_cap <= 4096;
    hipError_t e;
    if (whole) {
        e = select<4, VPR, PAGED>(a, keys, st);
        if (e != hipSuccess || a.new_len != a.cache_len) return e;
        hipLaunchKernelGGL(evict_lengths_kernel, dim3((a.B + 255) / 256), dim3(256), 0, st, a);
        return hipGetLastError();
    }
    e = few ? select<4, 0, PAGED>(a, keys, st) : select<16, 0, PAGED>(a, keys, st);
    if (e != hipSuccess) return e;
    const int rows = kMove / VPR * 4, most = (a.list_len + rows - 1) / rows;
    int runs = (32 * a.cus + units - 1) / units;          // (8 a CU: the last ones are waited for, 14 us of the above)
    if (runs > most) runs = most < 1 ? 1 : most;
    hipLaunchKernelGGL((evict_move_kernel<VPR, PAGED>), dim3((unsigned)units, (unsigned)runs), dim3(kMove), 0, st, a);
    return hipGetLastError();
}
template <int VPR>
hipError_t launch(const EvictArgs& a, hipStream_t st) {
    return a.block_table ? launch<VPR, true>(a, st) : launch<VPR, false>(a, st);
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
    switch (a.row_bytes / 16) {
        case 8: return launch<8>(a, st);
        case 16: return launch<16>(a, st);
        default: return launch<32>(a, st);
    }
}

}  // namespace s4c
