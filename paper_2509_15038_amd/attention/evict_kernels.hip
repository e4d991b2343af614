// Eviction by accumulated weight: of a head's L rows the `keep` best stay.
//     order: protected rows (the first and the most recent positions), then weight descending, then the lower row;
// rows below `keep` that stay keep their places, the holes among them are filled, in order, by the rows that stay from beyond: what moves is as few rows as leave,
// sources lie at or beyond `keep` and destinations below, so that a cache can be its own target with no order among the moves.
//
// evict_select_kernel, a workgroup a head: the newest position, how many rows are protected, the weight of the last row that stays by a radix search of four
// digits over order-preserving keys; then bitmaps in LDS, one bit a row, of the rows that stay and of those that tie with the last; all that is left
// (the first of the tied, ranks of holes and of those that fill them) are counts of bits.  evict_move_kernel copies rows, 16 bytes a lane.

#include <algorithm>
#include <type_traits>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Larger is better: weights in order, -0 as 0, NaN above all.
__device__ __forceinline__ uint32_t weight_key(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sums of x over the workgroup's threads, and the total.
__device__ __forceinline__ int before_me(int x, int* waves, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    __syncthreads();                   // (the last use of `waves`)
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return before + sum - x;
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

constexpr int kBins = 4096, kFineBins = 1024;      // 12 bits of a key, then 10, then 10
constexpr int kMostMoved = 128;                    // rows that the selection moves itself, in place

// Counts into bins; a wave whose lanes all count into one does so at once.
__device__ __forceinline__ void count_into(uint32_t* bins, uint32_t bin, bool counts) {
    const uint64_t who = __ballot(counts);
    if (!who) return;
    const uint32_t one = __builtin_amdgcn_readlane(bin, __builtin_ctzll(who));
    if (__ballot(counts && bin == one) == who) {
        if ((threadIdx.x & 63) == 0) atomicAdd(bins + one, (uint32_t)__popcll(who));
    } else if (counts) {
        atomicAdd(bins + bin, 1u);
    }
}

// A thread has rows tid, tid + 1024, ..: up to ROWS of them in registers, or, where the head is LONG, so many at a time, read again for every pass.
template <int ROWS, bool LONG>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictCall c) {
    extern __shared__ uint64_t bits[];                     // [words] rows that stay; [words] tied rows, then {those from beyond, holes} before the word
    uint32_t* bins = (uint32_t*)bits;                      // before that: [kBins] of the rows that are not protected, and that are; [kFineBins] of the last two digits
    __shared__ int waves[kWaves];
    __shared__ int newest_all, found_bin, found_need, many_moved;
    __shared__ int moved[kMostMoved][2];
    const int g = blockIdx.x, b = g / c.kv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n, stays = min(length, c.keep);
    const float* mass = c.mass + (int64_t)g * c.stride;
    const int32_t* positions = c.positions ? c.positions + (int64_t)g * c.stride : nullptr;
    int32_t* rows = c.rows + (int64_t)g * c.keep;
    float* mass_out = c.mass_out ? c.mass_out + (int64_t)g * c.out_stride : nullptr;
    int32_t* positions_out = c.positions_out ? c.positions_out + (int64_t)g * c.out_stride : nullptr;
    const auto place = [&](int i, int source) ALWAYS_INLINE {      // what goes with row i of the output
        rows[i] = source;
        if (mass_out && (mass_out != mass || source != i)) mass_out[i] = mass[source];
        if (positions_out && (positions_out != positions || source != i)) positions_out[i] = positions ? positions[source] : source;
    };
    for (int i = stays + tid; i < c.keep; i += kThreads) rows[i] = -1;
    if (length <= c.keep) {
        for (int i = tid; i < length; i += kThreads) place(i, i);
        return;
    }
    const int batches = LONG ? (length + ROWS * kThreads - 1) / (ROWS * kThreads) : 1;
    const auto row_of = [&](int batch, int k) ALWAYS_INLINE { return (batch * ROWS + k) * kThreads + tid; };
    for (int i = tid; i < 2 * kBins + 2 * kFineBins; i += kThreads) bins[i] = 0;
    if (tid == 0) newest_all = INT32_MIN, many_moved = 0;
    // The newest position.
    uint32_t key[ROWS];
    int at[ROWS], newest = INT32_MIN;
    const auto load_positions = [&](int batch) ALWAYS_INLINE {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int i = min(row_of(batch, k), length - 1);
            at[k] = positions ? positions[i] : i;
        }
    };
    const auto load_keys = [&](int batch) ALWAYS_INLINE {
        float x[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) x[k] = mass[min(row_of(batch, k), length - 1)];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) key[k] = weight_key(x[k]);
    };
    if (!LONG) load_keys(0);
    for (int batch = 0; batch < batches; ++batch) {
        load_positions(batch);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) newest = max(newest, at[k]);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) newest = max(newest, __shfl_xor(newest, d));
    __syncthreads();
    if (lane == 0) atomicMax(&newest_all, newest);
    __syncthreads();
    // Which of a thread's rows there are, and which are protected, a bit each.
    const int64_t after = (int64_t)newest_all - c.recent;
    uint32_t in = 0, first = 0;
    const auto look = [&](int batch) ALWAYS_INLINE {
        in = first = 0;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            in |= (uint32_t)(row_of(batch, k) < length) << k;
            first |= (uint32_t)(at[k] < c.sinks || at[k] > after) << k;
        }
    };
    if (!LONG) look(0);
    const auto each_batch = [&](auto&& what) ALWAYS_INLINE {
        for (int batch = 0; batch < batches; ++batch) {
            if (LONG) {
                load_positions(batch);
                load_keys(batch);
                look(batch);
            }
            what(batch);
        }
    };
    each_batch([&](int) ALWAYS_INLINE {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) count_into(bins, (key[k] >> 20) + (first >> k & 1) * kBins, in >> k & 1);
    });
    __syncthreads();
    // Among which rows the weight decides, how many of them stay, and the key of the last of these: the digit at which the count from the largest on reaches that many.
    int many_first;
    before_me((int)(bins[kBins + 4 * tid] + bins[kBins + 4 * tid + 1] + bins[kBins + 4 * tid + 2] + bins[kBins + 4 * tid + 3]), waves, &many_first);
    const bool among_first = many_first >= stays;
    int need = among_first ? stays : stays - many_first;
    const auto find = [&](const uint32_t* from, auto each) ALWAYS_INLINE {         // each: bins a thread, from the largest down
        constexpr int E = decltype(each)::value;
        const int top = E * kThreads - 1 - E * tid;
        int mine = 0, all;
#pragma unroll
        for (int i = 0; i < E; ++i) mine += from[top - i];
        int above = before_me(mine, waves, &all);
        if (above < need && above + mine >= need) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int count = from[top - i];
                if (above < need && above + count >= need) found_bin = top - i, found_need = need - above;
                above += count;
            }
        }
        __syncthreads();
        need = found_need;
        return (uint32_t)found_bin;
    };
    uint32_t last = find(bins + (among_first ? kBins : 0), std::integral_constant<int, 4>{});
#pragma unroll
    for (int digit = 0; digit < 2; ++digit) {
        uint32_t* fine = bins + 2 * kBins + digit * kFineBins;
        const int shift = 10 - 10 * digit;
        each_batch([&](int) ALWAYS_INLINE {
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                count_into(fine, key[k] >> shift & (kFineBins - 1), (in >> k & 1) && (first >> k & 1) == among_first && key[k] >> (shift + 10) == last);
        });
        __syncthreads();
        last = last << 10 | find(fine, std::integral_constant<int, 1>{});
    }
    // The bitmaps, and of the tied rows the first `need`.
    const int words = (length + 63) / 64;
    uint64_t* tied = bits + words;
    each_batch([&](int batch) ALWAYS_INLINE {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int w = (batch * ROWS + k) * kWaves + wave;
            const bool there = in >> k & 1, is_first = first >> k & 1;
            const uint64_t above = __ballot(there && (is_first == among_first ? key[k] > last : is_first)), ties = __ballot(there && is_first == among_first && key[k] == last);
            if (lane == 0 && w < words) bits[w] = above, tied[w] = ties;
        }
    });
    __syncthreads();
    const int each = (words + kThreads - 1) / kThreads, w0 = min(tid * each, words), w1 = min(w0 + each, words);
    int mine = 0, total;
    for (int w = w0; w < w1; ++w) mine += __popcll(tied[w]);
    int ahead = before_me(mine, waves, &total), holes = 0, beyond = 0;
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
    int holes_before = before_me(holes, waves, &total), beyond_before = before_me(beyond, waves, &total);
    u32x2* before = (u32x2*)tied;      // (a thread's own words)
    for (int w = w0; w < w1; ++w) {
        before[w] = (u32x2){(uint32_t)beyond_before, (uint32_t)holes_before};
        holes_before += __popcll(~bits[w] & low_of(w));
        beyond_before += __popcll(bits[w] & ~low_of(w));
    }
    __syncthreads();
    for (int i = tid; i < stays; i += kThreads) {
        const int w = i >> 6;
        const uint64_t x = bits[w], below = (1ull << (i & 63)) - 1;
        int source = i;
        if (!(x >> (i & 63) & 1)) {
            const uint32_t rank = before[w].y + __popcll(~x & below);
            int low = stays >> 6, high = words - 1;        // the last word with at most `rank` before it
            while (low < high) {
                const int mid = (low + high + 1) >> 1;
                if (before[mid].x <= rank) low = mid;
                else high = mid - 1;
            }
            source = low * 64 + bit_of_rank(bits[low] & ~low_of(low), rank - before[low].x);
            if (c.moves) {
                const int k = atomicAdd(&many_moved, 1);
                moved[k][0] = i, moved[k][1] = source;
            }
        }
        place(i, source);
    }
    if (!c.moves) return;
    __syncthreads();
    const int shift = c.dtype == CURDKV_DTYPE_BF16 ? 4 : 5;        // a row's pieces of 16 bytes; K, then V
    for (int i = tid; i < many_moved << (shift + 1); i += kThreads) {
        const int piece = i & ((1 << shift) - 1), k = i >> (shift + 1);
        u32x4a* array = (u32x4a*)(i >> shift & 1 ? c.V_out : c.K_out);
        array[(((int64_t)g * c.stride + moved[k][0]) << shift) + piece] = array[(((int64_t)g * c.stride + moved[k][1]) << shift) + piece];
    }
}

template <int LANES>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictCall c, int blocks) {
    constexpr int kRows = 256 / LANES;
    const int g = blockIdx.x / blocks, i = blockIdx.x % blocks * kRows + threadIdx.x / LANES, piece = threadIdx.x % LANES;
    if (i >= c.keep) return;
    const int source = c.rows[(int64_t)g * c.keep + i];
    if (source < 0 || (c.K_out == c.K && source == i)) return;
    const int64_t from = ((int64_t)g * c.stride + source) * LANES + piece, to = ((int64_t)g * c.out_stride + i) * LANES + piece;
    const u32x4a k = ((const u32x4a*)c.K)[from], v = ((const u32x4a*)c.V)[from];
    ((u32x4a*)c.K_out)[to] = k;
    ((u32x4a*)c.V_out)[to] = v;
}

}  // namespace

hipError_t launch_evict(const curdkv_ctx* ctx, const EvictCall& call, hipStream_t stream) {
    const unsigned heads = (unsigned)(call.count * call.kv);
    const size_t lds = std::max((size_t)((call.n + 63) / 64) * 16, (2 * kBins + 2 * kFineBins) * sizeof(uint32_t));
    EvictCall select = call;
    select.moves = call.K_out == call.K && call.n - call.keep <= kMostMoved;       // (in place; no more rows move than leave)
    const auto launch = [&](auto kernel) {
        const hipError_t e = lds <= 48 * 1024 ? hipSuccess : hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(kEvictMostRows / 64 * 16));
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
    // (at most 2^20 heads of 2^15 workgroups: whole heads a launch)
    for (unsigned h = 0; h < heads;) {
        const unsigned some = (unsigned)((kMostBlocks / blocks) < heads - h ? kMostBlocks / blocks : heads - h);
        EvictCall part = call;
        const int64_t row = bf16 ? 256 : 512;
        part.K += h * call.stride * row, part.V += h * call.stride * row;
        part.K_out += h * call.out_stride * row, part.V_out += h * call.out_stride * row;
        part.rows += (int64_t)h * call.keep;
        if (bf16) evict_move_kernel<16><<<some * blocks, 256, 0, stream>>>(part, blocks);
        else evict_move_kernel<32><<<some * blocks, 256, 0, stream>>>(part, blocks);
        h += some;
    }
    return hipGetLastError();
}

}  // namespace curdkv
