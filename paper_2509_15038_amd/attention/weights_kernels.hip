// The attention weight that every key of a cache got from a sequence's last m tokens, summed over them and the query heads of its KV head:
//     mass[j] = decay mass[j] + sum over rows R = (token, head) that see j of exp(scale q_R.k_j - lse_R),
// lse_R being the logarithm of the row's softmax denominator, which the attention has written.  With it no maximum has to be found: every weight is at
// most 1 (as far as lse is what the scores make it), and a key's sum is its own affair: one wave's, or a few waves' that are added up in order, without atomics.
//
// Few rows (weights_few_kernel): S = Q K^T by mfma_f32_16x16x32_bf16 (16x16x4 for fp32), 16 rows R by 16 keys; the rows stay in registers, a wave goes over keys.
// Many rows (weights_many_kernel): S^T = K Q^T by mfma_f32_32x32x16_bf16 (32x32x2); a wave's keys stay in registers, rows R go through LDS in stages of 16 KB that four waves
// share, and each lane adds up the weights of its own R, key by key, until all rows are through.

#include <algorithm>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

struct WeightsArgs {
    WeightsCall c;
    float scale_log2;
    int groups, rows, key_tiles;       // count * kv; m * group; tiles of keys a head
    int shares;                        // few rows: workgroups that share a head's keys
    int chunk, chunks;                 // many rows: that a workgroup takes
    float* part;                       // chunks > 1: [chunks][groups][key_tiles * keys of a tile], of the chunks that see some key of the tile
};

// Tokens of the m that see some key of j0 .. j1: [first, last].
struct Tokens {
    int first, last;
};
__device__ __forceinline__ Tokens tokens_that_see(int length, int m, int j0, int j1, int window, int sinks) {
    const int64_t p0 = (int64_t)length - m;                                                 // position of token 0
    const int64_t last = window > 0 && j0 >= sinks ? min((int64_t)m - 1, (int64_t)j1 + window - 1 - p0) : (int64_t)m - 1;
    return {(int)min(max((int64_t)j0 - p0, (int64_t)0), (int64_t)m), (int)max(last, (int64_t)-1)};
}
__device__ __forceinline__ int length_of(const WeightsCall& c, int b) { return __builtin_amdgcn_readfirstlane(c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n); }
__device__ __forceinline__ void add_to(const WeightsCall& c, int g, int j, float sum) {
    float* to = c.mass + (int64_t)g * c.mass_stride + j;
    *to = c.decay == 0.f ? sum : __builtin_fmaf(c.decay, *to, sum);
}

// ---- few rows

template <bool BF16> struct Operand;   // 128 channels of the row of lane % 16, those of the lane's quarter
template <> struct Operand<true> {
    u32x4a x[4];
    __device__ __forceinline__ void load(const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] = ((const u32x4a*)row)[4 * s + quarter];
    }
    static __device__ __forceinline__ f32x4a product(const Operand& a, const Operand& b) {
        f32x4a z = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < 4; ++s)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8a, a.x[s]), __builtin_bit_cast(bf16x8a, b.x[s]), z, 0, 0, 0);
        return z;
    }
};
template <> struct Operand<false> {
    f32x4a x[8];
    __device__ __forceinline__ void load(const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] = ((const f32x4a*)row)[4 * s + quarter];
    }
    static __device__ __forceinline__ f32x4a product(const Operand& a, const Operand& b) {
        f32x4a z = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[s][e], b.x[s][e], z, 0, 0, 0);
        return z;
    }
};

// Keys come in whole lines of 128 bytes: an instruction takes 8 rows' 8 pieces of 16 bytes, lane (quarter, c) piece quarter + 4 (c / 8) of row c % 8 of 8.  What the operand has in lane
// c < 8 from the second row of 8 and in lane c >= 8 from the first then lies 8 lanes off: x, of rows 0..7, and y, of rows 8..15, become pieces quarter and quarter + 4 of row c.
template <class T>
__device__ __forceinline__ void to_rows(T& x, T& y) {
    u32x4a u = __builtin_bit_cast(u32x4a, x), v = __builtin_bit_cast(u32x4a, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a = (int)u[i], b = (int)v[i];
        u[i] = (uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x128, 0xF, 0xC, false);       // row_ror:8, lanes 8..15 of 16
        v[i] = (uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x128, 0xF, 0x3, false);       // lanes 0..7
    }
    x = __builtin_bit_cast(T, u), y = __builtin_bit_cast(T, v);
}
#ifndef CM
#define CM 24
#endif
#ifndef CS
#define CS 2
#endif
#ifndef TE
#define TE 4
#endif
#ifndef AH
#define AH 1
#endif
#ifndef WV
#define WV 16
#endif

// 16 TILES rows R at most.  A wave takes the 64 keys of a step 16 at a time, kAhead more of them on their way, and reads and writes their weights together.
// PAST: keys pass the caches.
template <bool BF16, int TILES, bool PAST>
__global__ __launch_bounds__(256) void weights_few_kernel(WeightsArgs a) {
    constexpr int kRow = BF16 ? 256 : 512, kPieces = BF16 ? 4 : 8, kAhead = BF16 ? AH : 1;
    const WeightsCall& c = a.c;
    const int head = blockIdx.x % c.kv, share = blockIdx.x / c.kv % a.shares, b = blockIdx.x / c.kv / a.shares, g = b * c.kv + head;
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int length = length_of(c, b), steps = (length + 63) / 64;
    const int first = (int)((int64_t)steps * (share * 4 + wave) / (4 * a.shares)), end = (int)((int64_t)steps * (share * 4 + wave + 1) / (4 * a.shares));
    if (first >= end) return;
    const char* keys = (const char*)c.K + (int64_t)g * c.stride * kRow;
    float* mass = c.mass + (int64_t)g * c.mass_stride;
    Operand<BF16> ahead[4], q[TILES];
    const auto ask = [&](Operand<BF16>& k, int j0) ALWAYS_INLINE {
#pragma unroll
        for (int s = 0; s < kPieces; ++s) {
            const auto* from = (const decltype(k.x[s] + 0)*)(keys + (int64_t)min(j0 + (col & 7) + (s & 1) * 8, length - 1) * kRow + (quarter + (col >> 3) * 4 + (s >> 1) * 8) * 16);
            k.x[s] = PAST ? __builtin_nontemporal_load(from) : *from;
        }
    };
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ask(ahead[x], first * 64 + x * 16);
    // rows 16 u + col as the operand; of rows 16 u + 4 quarter + i, whose scores come back, the position (below all where the row gives nothing) and -lse
    int p[TILES][4];
    float less[TILES][4];
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        const int R = min(u * 16 + col, a.rows - 1);
        q[u].load((const char*)c.Q + ((((int64_t)b * c.m + R / c.group) * c.kv + head) * c.group + R % c.group) * kRow, quarter);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = u * 16 + 4 * quarter + i, at = min(r, a.rows - 1), token = at / c.group;
            const float lse = c.lse[((int64_t)b * c.kv * c.group + head * c.group + at % c.group) * c.m + token];
            p[u][i] = r < a.rows && lse != -INFINITY ? length - c.m + token : -1;
            less[u][i] = -lse * (1.f / kLn2);
        }
    }
    for (int step = first; step < end; ++step) {
        const int j = step * 64 + lane;
        const float old = mass[min(j, length - 1)];
        float mine = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            ask(ahead[(x + kAhead) % 4], step * 64 + (x + kAhead) * 16);
            Operand<BF16> k = ahead[x];
#pragma unroll
            for (int s = 0; s < kPieces; s += 2) to_rows(k.x[s], k.x[s + 1]);
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < TILES; ++u) {
                const f32x4a s = Operand<BF16>::product(q[u], k);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2, less[u][i]));
                    sum += sees(p[u][i], step * 64 + x * 16 + col, c.window, c.sinks) ? w : 0.f;
                }
            }
            sum = quarters_sum(sum);
            mine = quarter == x ? sum : mine;
        }
        if (j < length) mass[j] = c.decay == 0.f ? mine : __builtin_fmaf(c.decay, old, mine);
    }
}

// ---- many rows

// 64 lanes' 16 bytes, each from an address of its own, to LDS from `to` on (as dma16).
__device__ __forceinline__ void dma16_from(uint32_t to, const char* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}

template <bool BF16> struct Many;
template <> struct Many<true> {
    static constexpr int kBlocks = 2, kTiles = 4, kRow = 256;      // of 32 keys a wave; tiles of 32 rows a stage of 32 KB
    u32x4a x[8];
    __device__ __forceinline__ void load(const char* row, int half) {
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] = ((const u32x4a*)row)[2 * s + half];
    }
};
template <> struct Many<false> {
    static constexpr int kBlocks = 1, kTiles = 2, kRow = 512;
    f32x4a x[16];
    __device__ __forceinline__ void load(const char* row, int half) {
#pragma unroll
        for (int s = 0; s < 16; ++s) x[s] = ((const f32x4a*)row)[2 * s + half];
    }
};

// Where a row R = (token, head of the group) lies, moved on by `step` rows at a time without a division; units are the caller's.
struct Walk {
    int64_t at, step, wrap;            // step: of the whole tokens and the heads of a move; wrap: from a token's end to the next one's start
    int i, heads, group;
    __device__ __forceinline__ Walk(int R, int move, int group_, int64_t per_token, int64_t per_head)
        : at(R / group_ * per_token + R % group_ * per_head), step(move / group_ * per_token + move % group_ * per_head), wrap(per_token - group_ * per_head),
          i(R % group_), heads(move % group_), group(group_) {}
    __device__ __forceinline__ void on() {
        at += step;
        i += heads;
        if (i >= group) i -= group, at += wrap;
    }
};

// Sums of 2 W values over 2 W lanes, value `lane` to each lane's x[0]: at every step a lane keeps half of them and gives away the others'.
template <int W, int N>
__device__ __forceinline__ void spread(float (&x)[N], int lane) {
    const bool upper = lane & W;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float give = upper ? x[i] : x[i + W], keep = upper ? x[i + W] : x[i];
        x[i] = keep + __shfl_xor(give, W);
    }
    if constexpr (W > 1) spread<W / 2>(x, lane);
}

template <bool BF16>
__global__ __launch_bounds__(256, 2) void weights_many_kernel(WeightsArgs a) {
    typedef Many<BF16> M;
    constexpr int kKeys = M::kBlocks * 32, kTiles = M::kTiles, kStage = kTiles * 32;
    __shared__ __attribute__((aligned(16))) char Qs[2][32768];
    __shared__ float Ls[2][kStage];                                // -lse of a stage's rows, in units of log 2
    const WeightsCall& c = a.c;
    const int g = blockIdx.x % a.groups, key_tile = blockIdx.x / a.groups % a.key_tiles, chunk = blockIdx.x / a.groups / a.key_tiles, b = g / c.kv, head = g % c.kv;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int length = length_of(c, b), j0 = key_tile * (4 * kKeys), j1 = min(j0 + 4 * kKeys, length) - 1;
    if (j0 > j1) return;
    const Tokens seeing = tokens_that_see(length, c.m, j0, j1, c.window, c.sinks);
    const int begin = max(chunk * a.chunk, seeing.first * c.group / kStage * kStage), end = min(min((chunk + 1) * a.chunk, a.rows), (seeing.last + 1) * c.group);
    const int stages = (end - begin + kStage - 1) / kStage;        // (none: without parts the old weights may still have to fade)
    if (stages <= 0 && a.chunks > 1) return;

    // This wave's keys; the stages of which its keys are seen at all, and those whose rows all see all of them.
    const int k0 = j0 + wave * kKeys, k1 = min(k0 + kKeys, length) - 1;
    int seen_from = 0, seen_to = 0, whole_from = 0, whole_to = 0;
    if (k0 <= k1) {
        const Tokens some = tokens_that_see(length, c.m, k0, k1, c.window, c.sinks);
        seen_from = (max(some.first * c.group, begin) - begin) / kStage;
        seen_to = min(stages, ((some.last + 1) * c.group - begin + kStage - 1) / kStage);
        const int64_t all_first = max((int64_t)k1 - (length - c.m), (int64_t)0) * c.group;     // the first row that sees k1, and the first that does not see k0 any more
        const int64_t all_end = c.window > 0 && k1 >= c.sinks ? min((int64_t)a.rows, max((int64_t)k0 + c.window - (length - c.m), (int64_t)0) * c.group) : (int64_t)a.rows;
        whole_from = (int)min(max(all_first - begin + kStage - 1, (int64_t)0) / kStage, (int64_t)stages);
        whole_to = (int)min(max(all_end - begin, (int64_t)0) / kStage, (int64_t)stages);
        if (whole_to <= whole_from) whole_from = whole_to = stages;
    }
    M keys[M::kBlocks];
#pragma unroll
    for (int kb = 0; kb < M::kBlocks; ++kb) keys[kb].load((const char*)c.K + ((int64_t)g * c.stride + min(k0 + kb * 32 + col, length - 1)) * M::kRow, half);
    float sums[M::kBlocks * 16];
#pragma unroll
    for (int i = 0; i < M::kBlocks * 16; ++i) sums[i] = 0.f;

    // Rows on their way into LDS: tiles of 32 rows, in columns of 64 bytes a row, pieces of 16 permuted by (row / 2) % 4.  A wave has eight blocks of 16 rows' columns: of bf16 a
    // tile's, of fp32 half of a tile's.
    constexpr int kHalves = BF16 ? 2 : 1, kColumns = M::kRow / 64;
    const int tile_of = BF16 ? wave : wave >> 1, half_of = BF16 ? 0 : wave & 1, piece = (lane & 3) ^ ((lane >> 3) & 3);
    const int64_t per_token = (int64_t)c.kv * c.group * M::kRow, last_row = (a.rows - 1) / c.group * per_token + (c.group - 1) * M::kRow;
    const char* queries = (const char*)c.Q + ((int64_t)b * c.m * c.kv + head) * c.group * M::kRow + piece * 16;
    Walk low(begin + tile_of * 32 + half_of * 16 + (lane >> 2), kStage, c.group, per_token, M::kRow);
    Walk high(begin + tile_of * 32 + 16 + (lane >> 2), kStage, c.group, per_token, M::kRow);           // (bf16: the tile's other half)
    const float* lse_of_head = c.lse + ((int64_t)b * c.kv + head) * c.group * c.m;
    Walk less_of(begin + tid % kStage, kStage, c.group, 1, c.m);
    float next_less = 0.f;
    const uint32_t lds = lds_address(&Qs[0][0]) + tile_of * (kColumns * 2048) + half_of * 1024;
    const auto ask = [&](int stage) ALWAYS_INLINE {
        int64_t at[2] = {low.at, high.at}, l = less_of.at;
        if (begin + (stage + 1) * kStage > a.rows) {               // (what is behind the last row is not used)
            const int R = begin + stage * kStage + tile_of * 32 + half_of * 16 + (lane >> 2);
            if (R >= a.rows) at[0] = last_row;
            if (R + 16 >= a.rows) at[1] = last_row;
            if (begin + stage * kStage + tid % kStage >= a.rows) l = 0;
        }
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (stage & 1) * 32768);
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int i = 0; i < kColumns; ++i) dma16_from(to + h * 1024 + i * 2048, queries + at[h] + i * 64);
        next_less = lse_of_head[l];
        low.on();
        if (BF16) high.on();
        less_of.on();
    };
    const auto arrive = [&](int stage) ALWAYS_INLINE {
        if (tid < kStage) Ls[stage & 1][tid] = next_less == -INFINITY ? -INFINITY : -next_less * (1.f / kLn2);     // (a row that sees nothing weighs nothing)
        dma_wait();
        __syncthreads();
    };
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    // A stage of which some rows do not see some of the wave's keys, or are none.
    const auto masked_stage = [&](int stage) ALWAYS_INLINE {
#pragma unroll 1
        for (int u = 0; u < kTiles; ++u) {
            const int R = begin + stage * kStage + u * 32 + col;
            const float less = Ls[stage & 1][u * 32 + col];
            const int at = R < a.rows && less != -INFINITY ? length - c.m + R / c.group : -1;
            const char* Qt = Qs[stage & 1] + u * (kColumns * 2048);
#pragma unroll
            for (int kb = 0; kb < M::kBlocks; ++kb) {
                f32x16a x;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
                for (int i = 0; i < M::kRow / 32; ++i) {
                    const u32x4a q = *(const u32x4a*)(Qt + k_at[i & 1] + (i >> 1) * 2048);
                    if constexpr (BF16) {
                        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, keys[kb].x[i]), __builtin_bit_cast(bf16x8a, q), x, 0, 0, 0);
                    } else {
                        const f32x4a y = __builtin_bit_cast(f32x4a, q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(keys[kb].x[i][e], y[e], x, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less));
                    sums[kb * 16 + i] += sees(at, k0 + kb * 32 + i / 4 * 8 + i % 4 + half * 4, c.window, c.sinks) ? w : 0.f;
                }
            }
        }
    };
    if (stages > 0) {
        ask(0);
        arrive(0);
    }
    int stage = 0;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {                         // stages with masks, whole ones, some with masks again
        const int until = turn == 0 ? min(whole_from, stages) : stages;
#pragma unroll 1
        for (; stage < until; ++stage) {
            if (stage + 1 < stages) ask(stage + 1);
            if (stage >= seen_from && stage < seen_to) masked_stage(stage);
            if (stage + 1 < stages) arrive(stage + 1);
        }
        if (turn == 1 || stage >= whole_to) continue;
        if constexpr (BF16) {
            // The scores of the last block of 32 x 32 wait for the next one's products, between which their exponentials go.
            f32x16a s[2];
            float waiting = -INFINITY;                             // the -lse of s[1], of this wave's second 32 keys
#pragma unroll
            for (int i = 0; i < 16; ++i) s[1][i] = 0.f;
            const auto weigh = [&](const f32x16a& x, int kb, float less, int first, int count) ALWAYS_INLINE {
#pragma unroll
                for (int i = first; i < first + count; ++i) sums[kb * 16 + i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less));
            };
            u32x4a q[8];
            const auto read = [&](const char* Qt, int i) ALWAYS_INLINE { q[i] = *(const u32x4a*)(Qt + k_at[i & 1] + (i >> 1) * 2048); };
            const auto block = [&](int kb, f32x16a& x, const f32x16a& before, float less, const char* Qt) ALWAYS_INLINE {
                const f32x16a zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, keys[kb].x[i]), __builtin_bit_cast(bf16x8a, q[i]), i == 0 ? zero : x, 0, 0, 0);
                    if (kb == 1) read(Qt, i);                                      // (the next tile's)
                    __builtin_amdgcn_sched_barrier(0);
                    if (i == 1) weigh(before, 1 - kb, less, 0, 3);                 // (a product's results are not there at once)
                    if (i > 1 && i < 7) weigh(before, 1 - kb, less, 2 * i - 1, 2);
                    if (i == 7) weigh(before, 1 - kb, less, 13, 3);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
#pragma unroll 1
            for (; stage < whole_to; ++stage) {
                if (stage + 1 < stages) ask(stage + 1);
                const char* Qt = Qs[stage & 1];
#pragma unroll
                for (int i = 0; i < 8; ++i) read(Qt, i);
#pragma unroll 1
                for (int u = 0; u < kTiles; ++u) {
                    const float less = Ls[stage & 1][u * 32 + col];
                    Qt += u + 1 < kTiles ? kColumns * 2048 : 0;
                    block(0, s[0], s[1], waiting, Qt);
                    block(1, s[1], s[0], less, Qt);
                    waiting = less;
                }
                if (stage + 1 < stages) arrive(stage + 1);
            }
            weigh(s[1], 1, waiting, 0, 16);
        } else {
#pragma unroll 1
            for (; stage < whole_to; ++stage) {
                if (stage + 1 < stages) ask(stage + 1);
                masked_stage(stage);
                if (stage + 1 < stages) arrive(stage + 1);
            }
        }
    }
    if constexpr (!BF16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[i] += __shfl_xor(sums[i], 16);
    }
    spread<M::kBlocks * 8>(sums, col);
    const int i = col & 15, kb = BF16 ? col >> 4 : 0, j = k0 + kb * 32 + i / 4 * 8 + i % 4 + half * 4;
    if (j >= length || (!BF16 && col >= 16)) return;
    if (a.chunks > 1) a.part[((int64_t)chunk * a.groups + g) * a.key_tiles * (4 * kKeys) + j] = sums[0];
    else add_to(c, g, j, sums[0]);
}

// Adds up the chunks that see a key's tile, in order.
template <bool BF16>
__global__ __launch_bounds__(256) void weights_join_kernel(WeightsArgs a) {
    constexpr int kKeys = Many<BF16>::kBlocks * 128, kStage = Many<BF16>::kTiles * 32;
    const WeightsCall& c = a.c;
    const int g = blockIdx.x % a.groups, j = blockIdx.x / a.groups * 256 + threadIdx.x, length = length_of(c, g / c.kv);
    if (j >= length) return;
    const int j0 = j / kKeys * kKeys;
    const Tokens seeing = tokens_that_see(length, c.m, j0, min(j0 + kKeys, length) - 1, c.window, c.sinks);
    const int begin = seeing.first * c.group / kStage * kStage, end = min(a.rows, (seeing.last + 1) * c.group);
    float sum = 0.f;
    if (begin < end)
        for (int chunk = begin / a.chunk; chunk <= (end - 1) / a.chunk; ++chunk) sum += a.part[((int64_t)chunk * a.groups + g) * a.key_tiles * kKeys + j];
    add_to(c, g, j, sum);
}

}  // namespace

hipError_t launch_weights(const curdkv_ctx* ctx, const WeightsCall& call, hipStream_t stream) {
    const bool bf16 = call.dtype == CURDKV_DTYPE_BF16;
    WeightsArgs a{call, call.scale * (1.f / kLn2), (int)(call.count * call.kv), call.m * call.group, 0, 0, 0, 1, nullptr};
    if (a.rows <= 32) {
        const int64_t steps = (call.n + 63) / 64, waves = WV * (int64_t)ctx->num_cu;
        const int64_t each = std::max<int64_t>(1, std::min<int64_t>(TE, a.groups * steps / waves));
        a.shares = (int)((steps + 4 * each - 1) / (4 * each));
        const bool past = (int64_t)a.groups * call.n * (bf16 ? 256 : 512) > kPastCaches;
        const auto launch = [&](auto kernel) { kernel<<<(unsigned)((int64_t)a.groups * a.shares), 256, 0, stream>>>(a); };
        if (bf16 && a.rows <= 16) past ? launch(weights_few_kernel<true, 1, true>) : launch(weights_few_kernel<true, 1, false>);
        else if (bf16) past ? launch(weights_few_kernel<true, 2, true>) : launch(weights_few_kernel<true, 2, false>);
        else if (a.rows <= 16) past ? launch(weights_few_kernel<false, 1, true>) : launch(weights_few_kernel<false, 1, false>);
        else past ? launch(weights_few_kernel<false, 2, true>) : launch(weights_few_kernel<false, 2, false>);
        return hipGetLastError();
    }
    const int keys = bf16 ? 256 : 128, stage = bf16 ? 128 : 64;
    a.key_tiles = (call.n + keys - 1) / keys;
    // Rows shared out over workgroups until there are eight for every unit, half of them above the diagonal, eight stages each at least, as far as there is scratch.
    const int64_t blocks = (int64_t)a.groups * a.key_tiles, room = call.scratch ? (call.scratch_bytes - kScratchCounters) / (blocks * keys * (int64_t)sizeof(float)) : 0;
    const int64_t chunks = std::max<int64_t>(1, std::min(std::min<int64_t>(CM * (int64_t)ctx->num_cu / blocks, a.rows / (CS * stage)), std::min(room, kMostBlocks / blocks)));
    a.chunk = (int)(((a.rows + chunks - 1) / chunks + stage - 1) / stage * stage);
    a.chunks = (a.rows + a.chunk - 1) / a.chunk;
    a.part = (float*)((char*)call.scratch + kScratchCounters);
    const auto launch = [&](auto kernel, int64_t n) { kernel<<<(unsigned)n, 256, 0, stream>>>(a); };
    bf16 ? launch(weights_many_kernel<true>, blocks * a.chunks) : launch(weights_many_kernel<false>, blocks * a.chunks);
    if (a.chunks > 1) {
        const int64_t joins = (int64_t)a.groups * ((call.n + 255) / 256);
        bf16 ? launch(weights_join_kernel<true>, joins) : launch(weights_join_kernel<false>, joins);
    }
    return hipGetLastError();
}

}  // namespace curdkv
