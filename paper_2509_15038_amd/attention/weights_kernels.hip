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

// A row R as (token, head of the group), moved on without a division.
struct Row {
    int t, i;
    __device__ __forceinline__ Row() {}
    __device__ __forceinline__ Row(int R, int group) : t(R / group), i(R % group) {}
    __device__ __forceinline__ void on(int tokens, int heads, int group) {
        t += tokens, i += heads;
        if (i >= group) i -= group, ++t;
    }
};

template <bool BF16> struct Many;
template <> struct Many<true> {
    static constexpr int kBlocks = 2, kStage = 64, kRow = 256;     // of 32 keys a wave; rows a stage of 16 KB
    u32x4a x[8];
    __device__ __forceinline__ void load(const char* row, int half) {
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] = ((const u32x4a*)row)[2 * s + half];
    }
};
template <> struct Many<false> {
    static constexpr int kBlocks = 1, kStage = 32, kRow = 512;
    f32x4a x[16];
    __device__ __forceinline__ void load(const char* row, int half) {
#pragma unroll
        for (int s = 0; s < 16; ++s) x[s] = ((const f32x4a*)row)[2 * s + half];
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
    constexpr int kKeys = M::kBlocks * 32, kStage = M::kStage;
    __shared__ __attribute__((aligned(16))) char Qs[2][16384];
    const WeightsCall& c = a.c;
    const int g = blockIdx.x % a.groups, key_tile = blockIdx.x / a.groups % a.key_tiles, chunk = blockIdx.x / a.groups / a.key_tiles, b = g / c.kv, head = g % c.kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int length = length_of(c, b), j0 = key_tile * (4 * kKeys), j1 = min(j0 + 4 * kKeys, length) - 1;
    if (j0 > j1) return;
    const Tokens seeing = tokens_that_see(length, c.m, j0, j1, c.window, c.sinks);
    const int begin = max(chunk * a.chunk, seeing.first * c.group / kStage * kStage), end = min(min((chunk + 1) * a.chunk, a.rows), (seeing.last + 1) * c.group);
    const bool nothing = begin >= end;                             // (without parts the old weights may still have to fade)
    if (nothing && a.chunks > 1) return;

    const int k0 = j0 + wave * kKeys, k1 = min(k0 + kKeys, length) - 1;        // this wave's keys
    M keys[M::kBlocks];
#pragma unroll
    for (int kb = 0; kb < M::kBlocks; ++kb) keys[kb].load((const char*)c.K + ((int64_t)g * c.stride + min(k0 + kb * 32 + col, length - 1)) * M::kRow, half);
    float sums[M::kBlocks * 16];
#pragma unroll
    for (int i = 0; i < M::kBlocks * 16; ++i) sums[i] = 0.f;

    // Rows R on their way into LDS: columns of 64 bytes a row, pieces permuted by (row / 2) % 4; this lane's is row d_row of a stage, four columns of it from `column` on.
    const int64_t per_token = (int64_t)c.kv * c.group * M::kRow;
    const char* queries = (const char*)c.Q + ((int64_t)b * c.m * c.kv + head) * c.group * M::kRow;
    const int d_row = (BF16 ? wave : wave & 1) * 16 + (lane >> 2), column = BF16 ? 0 : (wave >> 1) * 4;
    const int piece = (lane & 3) ^ ((d_row >> 1) & 3);
    const int stage_tokens = kStage / c.group, stage_heads = kStage % c.group, last_t = (a.rows - 1) / c.group, last_i = c.group - 1;
    Row from(begin + d_row, c.group);
    const uint32_t lds = lds_address(&Qs[0][0]);
    const auto ask = [&](int buffer) ALWAYS_INLINE {
        const bool there = from.t <= last_t;
        const char* at = queries + (there ? from.t : last_t) * per_token + (there ? from.i : last_i) * M::kRow + column * 64 + piece * 16;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + buffer * 16384 + column * (kStage * 64) + (BF16 ? wave : wave & 1) * 1024);
#pragma unroll
        for (int i = 0; i < 4; ++i) dma16_from(to + i * (kStage * 64), at + i * 64);
        from.on(stage_tokens, stage_heads, c.group);
    };
    // The rows that this lane has scores of, R = 32 u + col of a stage: position and -lse.
    constexpr int kTiles = kStage / 32;
    const float* lse_of_head = c.lse + ((int64_t)b * c.kv + head) * c.group * c.m;
    Row mine[kTiles];
#pragma unroll
    for (int u = 0; u < kTiles; ++u) mine[u] = Row(begin + u * 32 + col, c.group);
    float lse[kTiles], next_lse[kTiles];
    int p[kTiles];
    const auto ask_lse = [&]() ALWAYS_INLINE {
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            const bool there = mine[u].t <= last_t;
            next_lse[u] = lse_of_head[(int64_t)(there ? mine[u].i : last_i) * c.m + (there ? mine[u].t : last_t)];
        }
    };
    if (!nothing) {
        ask(0);
        ask_lse();
        dma_wait();
    }
    __syncthreads();
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    // bf16: the scores of the last block of 32 x 32 wait for the next one's products, between which their exponentials go
    f32x16a s[2];
    float waiting = -INFINITY;                                     // the -lse of s[1], of this wave's second 32 keys
#pragma unroll
    for (int i = 0; i < 16; ++i) s[1][i] = 0.f;
    const auto weigh = [&](f32x16a& x, int kb, float less) ALWAYS_INLINE {
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[kb * 16 + i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less));
    };
    for (int R0 = begin, buffer = 0; R0 < end; R0 += kStage, buffer ^= 1) {
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            lse[u] = next_lse[u];
            p[u] = mine[u].t <= last_t ? length - c.m + mine[u].t : -1;
            mine[u].on(stage_tokens, stage_heads, c.group);
        }
        if (R0 + kStage < end) {
            ask(buffer ^ 1);
            ask_lse();
        }
        // positions of the stage's rows, lowest (in lane 0) and highest; rows that are none stand at -1
        const int low = __builtin_amdgcn_readfirstlane(p[0]), last = __builtin_amdgcn_readlane(p[kTiles - 1], 31), high = last < 0 ? length - 1 : last;
        const bool whole = last >= 0 && low >= k1 && (c.window <= 0 || high - k0 < c.window || k1 < c.sinks) && !__any(lse[0] == -INFINITY || lse[kTiles - 1] == -INFINITY);
        if (k0 > k1 || high < k0) {
        } else if (BF16 && whole) {
            if constexpr (BF16) {
                const auto block = [&](const u32x4a (&q)[8], int kb, f32x16a& x, f32x16a& before, int kb_before, float less) ALWAYS_INLINE {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const f32x16a zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
                        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, keys[kb].x[i]), __builtin_bit_cast(bf16x8a, q[i]), i == 0 ? zero : x, 0, 0, 0);
#pragma unroll
                        for (int e = 2 * i; e < 2 * i + 2; ++e) sums[kb_before * 16 + e] += __builtin_amdgcn_exp2f(__builtin_fmaf(before[e], a.scale_log2, less));
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
#pragma unroll
                for (int u = 0; u < kTiles; ++u) {
                    u32x4a q[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = *(const u32x4a*)(Qs[buffer] + u * 2048 + k_at[i & 1] + (i >> 1) * (kStage * 64));
                    const float less = -lse[u] * (1.f / kLn2);
                    block(q, 0, s[0], s[1], 1, waiting);
                    block(q, 1, s[1], s[0], 0, less);
                    waiting = less;
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < kTiles; ++u) {
                const int at = lse[u] == -INFINITY ? -1 : p[u];
                const float less = -lse[u] * (1.f / kLn2);
                const char* Qt = Qs[buffer] + u * 2048;
#pragma unroll
                for (int kb = 0; kb < M::kBlocks; ++kb) {
                    f32x16a x;
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
                    for (int i = 0; i < (BF16 ? 8 : 16); ++i) {
                        const u32x4a q = *(const u32x4a*)(Qt + k_at[i & 1] + (i >> 1) * (kStage * 64));
                        if constexpr (BF16) {
                            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, keys[kb].x[i]), __builtin_bit_cast(bf16x8a, q), x, 0, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(keys[kb].x[i][e], __uint_as_float(q[e]), x, 0, 0, 0);
                        }
                    }
                    if (!BF16 && whole) {
                        weigh(x, kb, less);
                        continue;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less));
                        sums[kb * 16 + i] += sees(at, k0 + kb * 32 + i / 4 * 8 + i % 4 + half * 4, c.window, c.sinks) ? w : 0.f;
                    }
                }
            }
        }
        dma_wait();
        __syncthreads();
    }
    if constexpr (BF16) weigh(s[1], 1, waiting);
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
    constexpr int kKeys = Many<BF16>::kBlocks * 128, kStage = Many<BF16>::kStage;
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
    const int keys = bf16 ? 256 : 128, stage = bf16 ? 64 : 32;
    a.key_tiles = (call.n + keys - 1) / keys;
    // Rows shared out over workgroups until there are eight for every unit, half of them above the diagonal, eight stages each at least, as far as there is scratch.
    const int64_t blocks = (int64_t)a.groups * a.key_tiles, room = call.scratch ? (call.scratch_bytes - kScratchCounters) / (blocks * keys * (int64_t)sizeof(float)) : 0;
    const int64_t chunks = std::max<int64_t>(1, std::min(std::min<int64_t>(16 * (int64_t)ctx->num_cu / blocks, a.rows / (8 * stage)), std::min(room, kMostBlocks / blocks)));
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
