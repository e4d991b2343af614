// Eviction by accumulated weight: of a head's L rows the `keep` best stay.
//     order: protected rows (the first and the most recent positions), then weight descending, then the lower row;
// rows below `keep` that stay keep their places, the holes among them are filled, in order, by the rows that stay from beyond: what moves is as few rows as leave,
// sources lie at or beyond `keep` and destinations below, so that a cache can be its own target with no order among the moves.
//
// evict_select_kernel, a workgroup a head.  A row's key is its weight's bits in an order that integers have, the largest for a protected row and 0 for what is none, so that the `keep`
// largest keys stay (should there be more protected rows, they have their weights' keys and all others 0).  The last key that stays is found digit by digit, 12 bits of all keys, then
// 10 and 10 of the few that share these.  Then bitmaps in LDS, one bit a row, of the rows that stay and of those that tie with the last; all that is left
// (the first of the tied, ranks of holes and of those that fill them) are counts of bits.  evict_move_kernel copies rows, 16 bytes a lane.
//
// Bound by: of many heads, the copy (128 heads of up to 16384 rows, 4096 of which stay and move: 495 MB, 107 us, of which the copy 90 at 5 TB/s); of few heads, one unit's vector
// instructions, of which one for every row takes 0.25 us at 32768 rows (8 heads, 10 % stay: 28 us, selection 21 and copy 6; 131072 rows 125 to 132); of a generated token, a chain of latencies
// and the launch (32 sequences of 8 heads, one of 3277 rows leaves each: 8.5 us).  That a head is one workgroup's is a choice: the call takes no scratch in which several could meet.  Heads of 16385
// to 32768 rows hold 32 rows a thread in the 128 registers that 1024 threads leave each, of which 5 spill (24 bytes a lane).

#include <algorithm>
#include <type_traits>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 4096, kFineBins = 1024;      // 12 bits of a key, then 10, then 10
constexpr int kListed = 2048;                      // keys of one bin that are kept apart
constexpr int kMostMoved = 128;                    // rows that the selection moves itself, in place (24 of 3300 of 256 heads 14.7 us, 53.6 by another kernel; 100 of 1001 of 64 heads 11.9, 15.3)
constexpr size_t kOwnLds = 24 * 1024;              // what the selection's arrays of fixed size take at most
constexpr int kFewLeave = 8;                       // rows that are found one by one (of 256 heads of some 3280: one 8.5 us, 13.6 by digits; four 10.3, 14.1; eight 11.0, 12.1)

// Larger is better: 0 for what is none, weights in order, -0 as 0, NaN above all, and above that the protected.
constexpr uint32_t kProtected = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t weight_key(float x) {
    if (x != x) return kProtected - 1;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum over the workgroup's threads below this one; `waves`: not used by the calls right before and after.
__device__ __forceinline__ int before_me(int x, int* waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sum = up_to(x);
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) before += w < wave ? waves[w] : 0;
    return before + sum - x;
}

// The smallest key of a wave's lanes, and the highest row that has it.
struct Worst {
    uint32_t key;
    int row;
};
template <int CTRL, int ROWS>
__device__ __forceinline__ void lower(uint32_t& x) { x = min(x, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)x, CTRL, ROWS, 0xF, false)); }
__device__ __forceinline__ uint32_t lowest(uint32_t x) {       // (as up_to)
    lower<0x111, 0xF>(x);
    lower<0x112, 0xF>(x);
    lower<0x114, 0xF>(x);
    lower<0x118, 0xF>(x);
    lower<0x142, 0xA>(x);
    lower<0x143, 0xC>(x);
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ Worst worst_of(uint32_t key, int row) {
    const uint32_t least = lowest(key);
    return {least, ~(int)lowest(key == least ? ~(uint32_t)row : ~0u)};
}

// By every wave alone: the largest x with at least `need` counted at x and above; `need` becomes how many of those at x are needed.  count(l): of lane l's, from the largest down.
struct Found {
    int lane, need;
};
template <class C>
__device__ __forceinline__ Found find(int need, const C& count) {
    const int mine = count((int)(threadIdx.x & 63)), sum = up_to(mine);
    const int lane = __builtin_ctzll(__ballot(sum >= need));
    return {lane, need - (__builtin_amdgcn_readlane(sum, lane) - __builtin_amdgcn_readlane(mine, lane))};
}

// The place of the set bit of x that has k set bits below it (k < their number).
__device__ __forceinline__ int bit_of_rank(uint64_t x, int k) {
    int at = 0;
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) {
        const int below = __popcll(x >> at & ((1ull << w) - 1));
        if (k >= below) k -= below, at += w;
    }
    return at;
}

// Four numbers that lie anywhere.
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));

// A thread has four rows in every 4096: up to ROWS of them in registers, or, where the head is LONG, so many at a time, read again for every pass.
template <int ROWS, bool LONG>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictCall c) {
    constexpr int kCopies = ROWS > 4 ? 2 : 1;              // of the first digit's bins, for neighbouring lanes (32768 rows: one 30.9 us, two 30.1, four 30.2)
    extern __shared__ __attribute__((aligned(16))) uint64_t bits[];                     // [words] rows that stay; [words] tied rows, then {those from beyond, holes} before the word; a list
    uint32_t* bins = (uint32_t*)bits;                      // before that
    __shared__ __attribute__((aligned(16))) uint32_t fine[2][kFineBins], listed[kListed];
    __shared__ int coarse[64], waves[3][kWaves];
    __shared__ int newest_all, many_first, many_listed, many_moved;
    __shared__ int moved[kMostMoved][2];
    const int g = blockIdx.x, b = g / c.kv, tid = threadIdx.x, lane = tid & 63;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n, stays = min(length, c.keep);
    const float* mass = c.mass + (int64_t)g * c.stride;
    const int32_t* positions = c.positions ? c.positions + (int64_t)g * c.stride : nullptr;
    int32_t* rows = c.rows + (int64_t)g * c.keep;
    float* mass_out = c.mass_out ? c.mass_out + (int64_t)g * c.out_stride : nullptr;
    int32_t* positions_out = c.positions_out ? c.positions_out + (int64_t)g * c.out_stride : nullptr;
    // what goes with rows i + 1024 e of the output (source < 0: nothing); where rows are moved by another kernel, that does it
    const auto place = [&](int i, const int (&source)[4]) ALWAYS_INLINE {
        float w[4];
        int p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int from = max(source[e], 0), to = i + e * kThreads;
            if (source[e] >= 0) rows[to] = from;
            if (!c.moves) continue;
            if (mass_out && (mass_out != mass || from != to)) w[e] = mass[from];
            if (positions_out && positions && (positions_out != positions || from != to)) p[e] = positions[from];
        }
        if (!c.moves) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int from = source[e], to = i + e * kThreads;
            if (from < 0) continue;
            if (mass_out && (mass_out != mass || from != to)) mass_out[to] = w[e];
            if (positions_out && (positions_out != positions || from != to)) positions_out[to] = positions ? p[e] : from;
        }
    };
    const auto move_rows = [&]() ALWAYS_INLINE {
        if (!c.moves) return;
        __syncthreads();
        const int shift = c.dtype == CURDKV_DTYPE_BF16 ? 4 : 5;        // a row's pieces of 16 bytes; K, then V
        for (int i = tid; i < many_moved << (shift + 1); i += kThreads) {
            const int piece = i & ((1 << shift) - 1), k = i >> (shift + 1);
            u32x4a* array = (u32x4a*)(i >> shift & 1 ? c.V_out : c.K_out);
            array[(((int64_t)g * c.stride + moved[k][0]) << shift) + piece] = array[(((int64_t)g * c.stride + moved[k][1]) << shift) + piece];
        }
    };
    for (int i = stays + tid; i < c.keep; i += kThreads) rows[i] = -1;
    if (length <= c.keep) {
        for (int i = tid; i < length; i += 4 * kThreads) {
            int source[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) source[e] = i + e * kThreads < length ? i + e * kThreads : -1;
            place(i, source);
        }
        return;
    }
    const int batches = LONG ? (length + ROWS * kThreads - 1) / (ROWS * kThreads) : 1;
    const auto row_of = [&](int batch, int k) ALWAYS_INLINE { return batch * (ROWS * kThreads) + (k / 4 * kThreads + tid) * 4 + k % 4; };
    // The newest position; meanwhile the bins are cleared.
    uint32_t key[ROWS];
    uint32_t at[ROWS], x[ROWS];
    int newest = INT32_MIN;
    const auto load = [&](const void* from, int batch, uint32_t* to) ALWAYS_INLINE {
#pragma unroll
        for (int k = 0; k < ROWS; k += 4) {
            const int i = row_of(batch, k);
            u32x4a y;
            if (i + 3 < length) {
                y = *(const u32x4u*)((const uint32_t*)from + i);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = ((const uint32_t*)from)[min(i + e, length - 1)];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) to[k + e] = y[e];
        }
    };
    const auto load_positions = [&](int batch) ALWAYS_INLINE {
        if (positions) load(positions, batch, at);
        else
#pragma unroll
            for (int k = 0; k < ROWS; ++k) at[k] = min(row_of(batch, k), length - 1);
    };
    const auto load_weights = [&](int batch) ALWAYS_INLINE { load(mass, batch, x); };
    if (!LONG) {
        load_positions(0);
        load_weights(0);
    }
    for (int i = tid; i < kBins * kCopies / 4; i += kThreads) ((u32x4a*)bins)[i] = (u32x4a){0, 0, 0, 0};
    fine[0][tid] = fine[1][tid] = 0;
    if (tid == 0) newest_all = INT32_MIN, many_first = many_listed = many_moved = 0;
    for (int batch = 0; batch < batches; ++batch) {
        if (LONG) load_positions(batch);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) newest = max(newest, (int)at[k]);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) newest = max(newest, __shfl_xor(newest, d));
    __syncthreads();
    if (lane == 0) atomicMax(&newest_all, newest);
    __syncthreads();
    // How many rows are protected: whose position, less the sinks, is not below `open`.
    const int from_on = (int)max((int64_t)newest_all - c.recent + (c.recent > 0), (int64_t)INT32_MIN);
    const uint32_t open = c.recent > 0 ? (uint32_t)max((int64_t)from_on - c.sinks, (int64_t)0) : 0x80000000u - (uint32_t)c.sinks;
    // (what the passes over the rows find is not kept from one to the next, as masks of 64 lanes it would fill more registers than there are)
    const auto apart = [&](uint32_t (&y)[ROWS]) ALWAYS_INLINE {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) loaded(y[k]);
    };
    // fours of rows of which all lanes have whole ones, and, otherwise, one by one those below `length`
    const auto each_row = [&](int batch, auto&& what, auto&& beyond) ALWAYS_INLINE {
        const int wave_row = batch * (ROWS * kThreads) + __builtin_amdgcn_readfirstlane(tid >> 6) * 256;
#pragma unroll
        for (int k = 0; k < ROWS; k += 4) {
            if (wave_row + k * kThreads + 256 <= length) {
#pragma unroll
                for (int e = 0; e < 4; ++e) what(k + e);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (row_of(batch, k + e) < length) what(k + e);
                    else beyond(k + e);
                }
            }
        }
    };
    int first = 0;
    for (int batch = 0; batch < batches; ++batch) {
        if (LONG) load_positions(batch);
        apart(at);
        each_row(batch, [&](int k) ALWAYS_INLINE { first += at[k] - (uint32_t)c.sinks >= open; }, [](int) {});
    }
    first = up_to(first);
    if (lane == 63) atomicAdd(&many_first, first);
    __syncthreads();
    const bool among_first = many_first > stays;
    int need = among_first ? stays : stays - many_first;           // of the rows whose weights decide
    const auto make_keys = [&](int batch) ALWAYS_INLINE {
        if (LONG) {
            load_positions(batch);
            load_weights(batch);
        }
        apart(at);
        each_row(batch, [&](int k) ALWAYS_INLINE {
            const uint32_t by_weight = weight_key(__uint_as_float(x[k]));
            const bool is_first = at[k] - (uint32_t)c.sinks >= open;
            if (among_first) key[k] = is_first ? by_weight : 0u;
            else key[k] = is_first ? kProtected : by_weight;
        }, [&](int k) ALWAYS_INLINE { key[k] = 0u; });
        apart(key);
    };
    if (!LONG) make_keys(0);
    const auto each_batch = [&](auto&& what) ALWAYS_INLINE {
        for (int batch = 0; batch < batches; ++batch) {
            if (LONG) make_keys(batch);
            what(batch);
            apart(key);
        }
    };
    const int leave = length - stays;
    if (!LONG && leave <= kFewLeave) {
        // Few leave: the smallest key of all, of equal ones the highest row, as often as that.
        __shared__ Worst worst[2][kWaves];
        int gone[kFewLeave] = {};
#pragma unroll
        for (int k = 0; k < ROWS; ++k) key[k] = row_of(0, k) < length ? key[k] : kProtected;
#pragma unroll
        for (int r = 0; r < kFewLeave; ++r) {
            if (r >= leave) continue;
            uint32_t least = kProtected;
            int row = 0;
#pragma unroll
            for (int k = 0; k < ROWS; ++k)                         // (rows ascending: the last of equal ones; what is none, or gone, has the largest key)
                if (key[k] <= least) least = key[k], row = row_of(0, k);
            const Worst mine = worst_of(least, row);
            if (lane == 0) worst[r & 1][tid >> 6] = mine;
            __syncthreads();
            const Worst of = worst[r & 1][lane & (kWaves - 1)];
            gone[r] = worst_of(of.key, of.row).row;
#pragma unroll
            for (int k = 0; k < ROWS; ++k) key[k] = row_of(0, k) == gone[r] ? kProtected : key[k];
        }
        // the k-th of those below `stays`, ascending, is the place of the k-th row from there on that is none of them
        const auto is_gone = [&](int i) ALWAYS_INLINE {
            bool y = false;
#pragma unroll
            for (int q = 0; q < kFewLeave; ++q) y |= q < leave && gone[q] == i;
            return y;
        };
        for (int i0 = tid; i0 < stays; i0 += 4 * kThreads) {
            int source[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + e * kThreads;
                source[e] = i < stays ? i : -1;
                if (i >= stays || !is_gone(i)) continue;
                int rank = 0;
#pragma unroll
                for (int q = 0; q < kFewLeave; ++q) rank += q < leave && gone[q] < i;
                for (int j = stays; j < length; ++j)
                    if (!is_gone(j) && rank-- == 0) source[e] = j;
                if (c.moves) {
                    const int k = atomicAdd(&many_moved, 1);
                    moved[k][0] = i, moved[k][1] = source[e];
                }
            }
            place(i0, source);
        }
        move_rows();
        return;
    }
    uint32_t last = kProtected - 1;                                // the last key that stays; where the protected are all that do, above it
    if (need > 0) {
        each_batch([&](int) ALWAYS_INLINE {
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                if (key[k] - 1 < kProtected - 1) atomicAdd(bins + (key[k] >> 20) * kCopies + (lane & (kCopies - 1)), 1u);
        });
        __syncthreads();
        int four = 0;                                              // of bins 4 tid .. 4 tid + 3, and then of 64 bins
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const u32x4a y = ((const u32x4a*)bins)[tid * kCopies + i];
            four += y[0] + y[1] + y[2] + y[3];
        }
        four += moved_by<0x111, 0xF>(four);
        four += moved_by<0x112, 0xF>(four);
        four += moved_by<0x114, 0xF>(four);
        four += moved_by<0x118, 0xF>(four);
        if ((lane & 15) == 15) coarse[tid >> 4] = four;
        __syncthreads();
        Found f = find(need, [&](int l) { return coarse[63 - l]; });
        const int top = (63 - f.lane) * 64 + 63;
        const auto in_bin = [&](int bin) {
            int sum = 0;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) sum += bins[bin * kCopies + i];
            return sum;
        };
        f = find(f.need, [&](int l) { return in_bin(top - l); });
        last = top - f.lane;
        need = f.need;
        const bool few = in_bin(last) <= kListed;
        if (few) {
            const uint32_t low = max(last << 20, 1u), span = min(last << 20 | 0xFFFFFu, kProtected - 1) - low;
            each_batch([&](int) ALWAYS_INLINE {
#pragma unroll
                for (int k = 0; k < ROWS; k += 4) {
                    if (min(min(key[k] - low, key[k + 1] - low), min(key[k + 2] - low, key[k + 3] - low)) > span) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key[k + e] - low <= span) listed[atomicAdd(&many_listed, 1)] = key[k + e];
                }
            });
            __syncthreads();
        }
        const int many = many_listed;
#pragma unroll
        for (int digit = 0; digit < 2; ++digit) {
            const int shift = 10 - 10 * digit;
            const auto count = [&](uint32_t k) ALWAYS_INLINE {
                if (k >> (shift + 10) == last && k - 1 < kProtected - 1) atomicAdd(fine[digit] + (k >> shift & (kFineBins - 1)), 1u);
            };
            if (few) {
                for (int i = tid; i < many; i += kThreads) count(listed[i]);
            } else {
                each_batch([&](int) ALWAYS_INLINE {
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) count(key[k]);
                });
            }
            __syncthreads();
            f = find(need, [&](int l) {
                int sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x4a y = ((const u32x4a*)fine[digit])[(63 - l) * 4 + i];
                    sum += y[0] + y[1] + y[2] + y[3];
                }
                return sum;
            });
            const int of16 = (63 - f.lane) * 16 + 15;
            f = find(f.need, [&](int l) { return l < 16 ? (int)fine[digit][of16 - l] : 0; });
            last = last << 10 | (of16 - f.lane);
            need = f.need;
        }
    }
    // The bitmaps, four lanes' rows written together, and of the tied rows the first `need`.
    const int words = (length + 63) / 64;
    uint64_t* tied = bits + words;
    __syncthreads();                                               // (nobody reads bins any more)
    each_batch([&](int batch) ALWAYS_INLINE {
#pragma unroll
        for (int k = 0; k < ROWS; k += 4) {
            uint32_t y = 0;                                        // above, and 16 bits on, tied
#pragma unroll
            for (int e = 0; e < 4; ++e) y |= (key[k + e] > last ? 1u << e : 0u) | (key[k + e] == last ? 0x10000u << e : 0u);
            y <<= (lane & 3) * 4;
            y |= (uint32_t)moved_by<0xB1, 0xF>((int)y);            // (quad_perm: xor 1, xor 2)
            y |= (uint32_t)moved_by<0x4E, 0xF>((int)y);
            const int sixteen = row_of(batch, k) >> 4;
            if ((lane & 3) == 0 && sixteen < words * 4) ((uint16_t*)bits)[sixteen] = (uint16_t)y, ((uint16_t*)tied)[sixteen] = (uint16_t)(y >> 16);
        }
    });
    __syncthreads();
    const int each = (words + kThreads - 1) / kThreads, w0 = min(tid * each, words), w1 = min(w0 + each, words);
    int mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popcll(tied[w]);
    int ahead = before_me(mine, waves[0]), holes = 0, beyond = 0;
    const auto low_of = [&](int w) ALWAYS_INLINE { return stays >= w * 64 + 64 ? ~0ull : stays <= w * 64 ? 0ull : (1ull << (stays - w * 64)) - 1; };   // rows below stays
    for (int w = w0; w < w1; ++w) {
        uint64_t x = tied[w];
        const int there = __popcll(x), take = min(max(need - ahead, 0), there);
        if (take < there) x = take ? x & ((2ull << bit_of_rank(x, take - 1)) - 1) : 0;
        ahead += there;
        bits[w] |= x;
        holes += __popcll(~bits[w] & low_of(w));
        beyond += __popcll(bits[w] & ~low_of(w));
    }
    int holes_before = before_me(holes, waves[1]), beyond_before = before_me(beyond, waves[2]);
    u32x2* before = (u32x2*)tied;      // (a thread's own words)
    for (int w = w0; w < w1; ++w) {
        before[w] = (u32x2){(uint32_t)beyond_before, (uint32_t)holes_before};
        holes_before += __popcll(~bits[w] & low_of(w));
        beyond_before += __popcll(bits[w] & ~low_of(w));
    }
    __syncthreads();
    // The rows from beyond, by rank: a list of them, or, where that has no room, looked for by the words' counts.
    uint16_t* from_beyond = (uint16_t*)(bits + 2 * words);
    if constexpr (!LONG) {
        const int w = tid >> 1, upper = tid & 1;
        if (w < words) {
            const uint64_t x = bits[w] & ~low_of(w);
            uint32_t mine = (uint32_t)(x >> (32 * upper)), rank = before[w].x + (upper ? __popc((uint32_t)x) : 0);
            for (; mine; mine &= mine - 1) from_beyond[rank++] = (uint16_t)(w * 64 + upper * 32 + __builtin_ctz(mine));
        }
        __syncthreads();
    }
    int step = 1;                                                  // the largest power of two below `words`
    while (step * 2 < words) step *= 2;
    for (int i0 = tid; i0 < stays; i0 += 4 * kThreads) {
        int source[4], low[4];
        uint32_t rank[4];
        bool hole[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + e * kThreads, w = min(i, stays - 1) >> 6;
            const uint64_t x = bits[w];
            hole[e] = i < stays && !(x >> (i & 63) & 1);
            rank[e] = before[w].y + __popcll(~x & ((1ull << (i & 63)) - 1));
            source[e] = i < stays ? i : -1;
            low[e] = 0;
        }
        for (int d = LONG ? step : 0; d > 0; d >>= 1)              // the last word with at most `rank` from beyond before it
#pragma unroll
            for (int e = 0; e < 4; ++e) low[e] += low[e] + d < words && before[min(low[e] + d, words - 1)].x <= rank[e] ? d : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!hole[e]) continue;
            source[e] = LONG ? low[e] * 64 + bit_of_rank(bits[low[e]] & ~low_of(low[e]), rank[e] - before[low[e]].x) : from_beyond[rank[e]];
            if (c.moves) {
                const int k = atomicAdd(&many_moved, 1);
                moved[k][0] = i0 + e * kThreads, moved[k][1] = source[e];
            }
        }
        place(i0, source);
    }
    move_rows();
}

template <int LANES>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictCall c, int blocks) {
    constexpr int kRows = 256 / LANES;
    const int g = blockIdx.x / blocks, i = blockIdx.x % blocks * kRows + threadIdx.x / LANES, piece = threadIdx.x % LANES;
    if (i >= c.keep) return;
    const int source = c.rows[(int64_t)g * c.keep + i];
    if (source < 0) return;
    if (piece == 0 && c.mass_out && (c.mass_out != c.mass || source != i)) c.mass_out[(int64_t)g * c.out_stride + i] = c.mass[(int64_t)g * c.stride + source];
    if (piece == 1 && c.positions_out && (c.positions_out != c.positions || source != i))
        c.positions_out[(int64_t)g * c.out_stride + i] = c.positions ? c.positions[(int64_t)g * c.stride + source] : source;
    if (c.K_out == c.K && source == i) return;
    const int64_t from = ((int64_t)g * c.stride + source) * LANES + piece, to = ((int64_t)g * c.out_stride + i) * LANES + piece;
    const u32x4a k = ((const u32x4a*)c.K)[from], v = ((const u32x4a*)c.V)[from];
    ((u32x4a*)c.K_out)[to] = k;
    ((u32x4a*)c.V_out)[to] = v;
}

}  // namespace

hipError_t launch_evict(const curdkv_ctx* ctx, const EvictCall& call, hipStream_t stream) {
    const unsigned heads = (unsigned)(call.count * call.kv);
    const bool is_long = call.n > 32 * kThreads;
    const int64_t most_moved = call.n > call.keep ? std::min<int64_t>(call.n - call.keep, call.keep) : 0;
    const size_t lds = std::max((size_t)((call.n + 63) / 64) * 16 + (is_long ? 0 : most_moved * 2), kBins * (call.n > 4 * kThreads ? 2 : 1) * sizeof(uint32_t));
    EvictCall select = call;
    select.moves = call.K_out == call.K && call.n - call.keep <= kMostMoved;       // (in place; no more rows move than leave)
    const auto launch = [&](auto kernel) {
        // (with the kernel's own arrays, 17.7 KB, a launch of up to 64 KB needs no leave for more: heads of up to 163840 rows)
        const hipError_t e = lds + kOwnLds <= 64 * 1024 ? hipSuccess : hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(kEvictMostRows / 64 * 16));
        if (e == hipSuccess) kernel<<<heads, kThreads, lds, stream>>>(select);
        return e;
    };
    const hipError_t e = call.n <= 4 * kThreads ? launch(evict_select_kernel<4, false>) : call.n <= 8 * kThreads ? launch(evict_select_kernel<8, false>)
                         : call.n <= 16 * kThreads ? launch(evict_select_kernel<16, false>) : call.n <= 32 * kThreads ? launch(evict_select_kernel<32, false>)
                                                                                              : launch(evict_select_kernel<16, true>);
    if (e != hipSuccess) return e;
    if (select.moves) return hipGetLastError();
    const int keep = call.keep < call.n ? call.keep : call.n;
    const bool bf16 = call.dtype == CURDKV_DTYPE_BF16;
    const int blocks = bf16 ? (keep + 15) / 16 : (keep + 7) / 8;
    // (at most 2^20 heads of 2^15 workgroups, in fp32 2^16: whole heads a launch)
    for (unsigned h = 0; h < heads;) {
        const unsigned some = (unsigned)((kMostBlocks / blocks) < heads - h ? kMostBlocks / blocks : heads - h);
        EvictCall part = call;
        const int64_t row = bf16 ? 256 : 512;
        part.K += h * call.stride * row, part.V += h * call.stride * row;
        part.K_out += h * call.out_stride * row, part.V_out += h * call.out_stride * row;
        part.rows += (int64_t)h * call.keep;
        part.mass += h * call.stride;
        if (part.mass_out) part.mass_out += h * call.out_stride;
        if (part.positions) part.positions += h * call.stride;
        if (part.positions_out) part.positions_out += h * call.out_stride;
        if (bf16) evict_move_kernel<16><<<some * blocks, 256, 0, stream>>>(part, blocks);
        else evict_move_kernel<32><<<some * blocks, 256, 0, stream>>>(part, blocks);
        h += some;
    }
    return hipGetLastError();
}

}  // namespace curdkv
