// Eviction by accumulated weight: of a head's L rows the `keep` best stay.
//     order: protected rows (the first and the most recent positions), then weight descending, then the lower row;
// rows below `keep` that stay keep their places, the holes among them are filled, in order, by the rows that stay from beyond: what moves is as few rows as leave,
// sources lie at or beyond `keep` and destinations below, so that a cache can be its own target with no order among the moves.
//
// evict_select_kernel, a workgroup a head: the newest position, how many rows are protected, the weight of the last row that stays by a radix search of four
// digits over order-preserving keys; then bitmaps in LDS, one bit a row, of the rows that stay and of those that tie with the last; all that is left
// (the first of the tied, ranks of holes and of those that fill them) are counts of bits.  evict_move_kernel copies rows, 16 bytes a lane.

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

__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictCall c) {
    extern __shared__ uint64_t bits[];                     // [words] rows that stay; [words] tied rows, then {those from beyond, holes} before the word
    __shared__ uint32_t hist[kWaves][256];
    __shared__ int waves[kWaves];
    __shared__ int newest_all, many_first, found_bin, found_need;
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
    // The newest position, and how many rows are protected.
    if (tid == 0) newest_all = INT32_MIN, many_first = 0;
    __syncthreads();
    int newest = INT32_MIN;
    if (!positions) newest = length - 1;
    else for (int i = tid; i < length; i += kThreads) newest = max(newest, positions[i]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) newest = max(newest, __shfl_xor(newest, d));
    if (lane == 0) atomicMax(&newest_all, newest);
    __syncthreads();
    const int64_t after = (int64_t)newest_all - c.recent;
    const auto protects = [&](int i) ALWAYS_INLINE {
        const int p = positions ? positions[i] : i;
        return p < c.sinks || p > after;
    };
    int first = 0;
    for (int i = tid; i < length; i += kThreads) first += protects(i);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) first += __shfl_xor(first, d);
    if (lane == 0) atomicAdd(&many_first, first);
    __syncthreads();
    // Among which rows the weight decides, how many of them stay, and the key of the last of these.
    const bool among_first = many_first >= stays;
    int need = among_first ? stays : stays - many_first;
    uint32_t last = 0, known = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < kWaves * 256; i += kThreads) (&hist[0][0])[i] = 0;
        __syncthreads();
        for (int i = tid; i < length; i += kThreads) {
            const uint32_t key = weight_key(mass[i]);
            if (protects(i) == among_first && (key & known) == last) atomicAdd(&hist[wave][key >> shift & 255], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            // lane l has bins 255 - 4 l .. 252 - 4 l, so that sums run from the largest digit on
            int count[4], mine = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                count[i] = 0;
                for (int w = 0; w < kWaves; ++w) count[i] += hist[w][255 - 4 * lane - i];
                mine += count[i];
            }
            int sum = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int y = __shfl_up(sum, d);
                if (lane >= d) sum += y;
            }
            int above = sum - mine;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (above < need && above + count[i] >= need) found_bin = 255 - 4 * lane - i, found_need = need - above;
                above += count[i];
            }
        }
        __syncthreads();
        last |= (uint32_t)found_bin << shift;
        known |= 255u << shift;
        need = found_need;             // (rows of the last key that stay, in the end)
        __syncthreads();
    }
    // The bitmaps, and of the tied rows the first `need`.
    const int words = (length + 63) / 64;
    uint64_t* tied = bits + words;
    for (int w = wave; w < words; w += kWaves) {
        const int i = w * 64 + lane, at = min(i, length - 1);
        const uint32_t key = weight_key(mass[at]);
        const bool is_first = protects(at), in = i < length;
        const uint64_t above = __ballot(in && (is_first == among_first ? key > last : is_first)), ties = __ballot(in && is_first == among_first && key == last);
        if (lane == 0) bits[w] = above, tied[w] = ties;
    }
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
        }
        place(i, source);
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
    const size_t lds = (size_t)((call.n + 63) / 64) * 16;
    const hipError_t e = lds <= 40 * 1024 ? hipSuccess
                                          : hipFuncSetAttribute((const void*)evict_select_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(kEvictMostRows / 64 * 16));
    if (e != hipSuccess) return e;
    evict_select_kernel<<<heads, kThreads, lds, stream>>>(call);
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
