// The attention weight that every key of a cache got from a sequence's last m tokens, summed over them and the query heads of its KV head:
//     mass[j] = decay mass[j] + sum over rows R = (token, head) that see j of exp(scale q_R.k_j - lse_R),
// lse_R being the logarithm of the row's softmax denominator, which the attention has written.  With it no maximum has to be found: every weight is at
// most 1 (as far as lse is what the scores make it), and a key's sum is its own affair: one wave's, or a few waves' that are added up in order, without atomics.
//
// Few rows, up to 32 of fp32 or over keys that pass the caches, up to 16 over few keys (weights_few_kernel): S = Q K^T by mfma_f32_16x16x32_bf16 (16x16x4 for fp32), 16 rows R by 16 keys; the rows stay in registers, a
// wave goes over keys, whose lines it reads whole.
// Up to 128 rows (weights_some_kernel): S^T = K Q^T by mfma_f32_32x32x16_bf16, 32 keys by 32 rows R; the rows stay in LDS, a wave goes over keys; each lane adds up the weights of its own R, key
// by key.
// Many rows (weights_many_kernel): the same (fp32: six products of parts); a wave's keys stay in registers, rows R go through LDS in stages of 16 KB that four waves share.
//
// Which of them: one token over 4097 keys of 8 heads 5.2 us by the first and 5.7 by the second, over 32768 16.5 and 13.8; 8 tokens' 32 rows 17.9 and 13.1 (by the third 20.3); over 131072 keys,
// past the caches, 46 and 56; 32 tokens over 32768 19 by the second, 23 by the third.  Keys that a window hides from all rows are not read (a token over 131072 with a window of 4096: 13 us).
// Bound by: few rows, HBM (a token of 32 sequences over up to 4096 rows, 137 MB, 31 us, 4.4 TB/s; one over 131072, 268 MB, 46 us, 5.8); up to 128, HBM at 4.4 TB/s after 3 us of start (32
// tokens over 32768 keys, 67 MB, 19 us); many rows, products and exponentials that wait for each other (a 128 by 64 block has 2048 clocks of products and some 2900 of exponentials and
// sums, of which little is at the same time: the matrix units are busy for 46 % of the clocks) and, for a seventh, the power that lowers the clock to 2.0 to 2.1 GHz: a prompt of 8192 tokens,
// 32 heads, 275 GFLOP, 280 to 290 us, 950 to 980 TFLOP/s (with zeros for numbers 244).  128 tokens over 32768 keys, 34 GFLOP, 49 us: a workgroup a tile of keys, 1024 of them two at a time
// on a unit, each of which loads its keys and goes over four stages, with nothing on its way for the next.  fp32 (three ragged prompts of up to 1021 tokens, window 257) 31.5 us: a workgroup's
// few stages each wait for their rows, are taken apart and meet two barriers, there being room for one stage.  Generated tokens in fp32: 32 sequences over up to 4096 rows, 270 MB, 61 us, 4.4
// TB/s; one over 131072, 545 MB, 105 us, 5.2.
// Each weight is rounded nowhere: scores, exponentials and sums are of 32 bits.

#include <algorithm>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

struct WeightsArgs {
    WeightsCall c;
    float scale_log2;
    int groups, rows, key_tiles;       // count * kv; m * group; tiles of keys a head
    int shares;                        // workgroups that share a head's keys; of many rows: its products (0: a workgroup has a tile of keys)
    int most;                          // many rows: stages whose queries lie within 2^31 bytes
    float* part;                       // many rows, shared: [groups][shares + key_tiles][keys of a tile], of share s and tile t at s + t, which no other pair has
    Divisor by_groups, by_kv, by_group;
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
// Whether any of the m tokens sees one of keys j0 .. j1 (below the length): the first one's window reaches lowest.
__device__ __forceinline__ bool any_sees(const WeightsCall& c, int length, int j0, int j1) { return (c.window == 0) | (j0 < c.sinks) | (c.window > length - c.m - j1); }
__device__ __forceinline__ void add_to(const WeightsCall& c, int g, int j, float sum, float decay) {
    float* to = c.mass + (int64_t)g * c.mass_stride + j;
    *to = decay == 0.f ? sum : __builtin_fmaf(decay, *to, sum);
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
// 16 TILES rows R at most.  A wave takes the 64 keys of a step 16 at a time, the next 16 on their way, and reads and writes their weights together.
// PAST: keys pass the caches (268 MB of them 47 us, 55 through the caches; 67 MB 17.8 and 16.5).
template <bool BF16, int TILES, bool PAST>
__global__ __launch_bounds__(256) void weights_few_kernel(WeightsArgs a) {
    constexpr int kRow = BF16 ? 256 : 512, kPieces = BF16 ? 4 : 8;
    const WeightsCall& c = a.c;
    const int head = blockIdx.x % c.kv, share = blockIdx.x / c.kv % a.shares, b = blockIdx.x / c.kv / a.shares, g = b * c.kv + head;
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int length = length_of(c, b), steps = (length + 63) / 64;
    const int first = (int)((int64_t)steps * (share * 4 + wave) / (4 * a.shares)), end = (int)((int64_t)steps * (share * 4 + wave + 1) / (4 * a.shares));
    if (first >= end) return;
    const char* keys = (const char*)c.K + (int64_t)g * c.stride * kRow;
    float* mass = c.mass + (int64_t)g * c.mass_stride;
    Operand<BF16> ahead[2], q[TILES];
    const auto ask = [&](Operand<BF16>& k, int j0) ALWAYS_INLINE {
#pragma unroll
        for (int s = 0; s < kPieces; ++s) {
            const auto* from = (const decltype(k.x[s] + 0)*)(keys + (int64_t)min(j0 + (col & 7) + (s & 1) * 8, length - 1) * kRow + (quarter + (col >> 3) * 4 + (s >> 1) * 8) * 16);
            k.x[s] = PAST ? __builtin_nontemporal_load(from) : *from;
        }
    };
    if (any_sees(c, length, first * 64, first * 64 + 63)) ask(ahead[0], first * 64);
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
        const bool seen = any_sees(c, length, step * 64, step * 64 + 63);
        const float old = seen || c.decay != 1.f ? mass[min(j, length - 1)] : 0.f;
        float mine = 0.f;
        if (!seen) {
            if (j < length && c.decay != 1.f) mass[j] = c.decay == 0.f ? 0.f : c.decay * old;
            if (any_sees(c, length, step * 64 + 64, step * 64 + 127)) ask(ahead[0], step * 64 + 64);
            continue;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            ask(ahead[(x + 1) % 2], step * 64 + x * 16 + 16);
            Operand<BF16> k = ahead[x % 2];
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

template <bool BF16> struct Many;
template <> struct Many<true> {
    static constexpr int kBlocks = 2, kTiles = 4, kRow = 256;      // of 32 keys a wave; tiles of 32 rows a stage of 32 KB
    u32x4a x[8];
    __device__ __forceinline__ void load(const char* row, int half) {
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] = ((const u32x4a*)row)[2 * s + half];
    }
};
// fp32: a number x is three of 8 bits, x = h + m + l exactly (h its upper half, m what is left rounded to bf16, l the rest, whose last bits end at 2^-133); of the nine products of parts the
// six that count go through the bf16 units, and what is left out is below 2^-22 of a product (2000 tokens over 2000, 16 GFLOP: 115 us, by products of 32 bits 164).  Infinities and NaN are h
// alone, and what holds one goes through products of 32 bits.
struct Parts {                         // of eight channels
    u32x4a h, m, l;
};
__device__ __forceinline__ Parts parts_of(f32x4a x, f32x4a y, bool& odd) {
    Parts p;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = i < 2 ? x[2 * i] : y[2 * i - 4], b = i < 2 ? x[2 * i + 1] : y[2 * i - 3];
        const uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
        most = max(most, max(u & 0x7FFFFFFFu, v & 0x7FFFFFFFu));
        p.h[i] = __builtin_amdgcn_perm(v, u, 0x07060302u);
        const float r = a - __uint_as_float(u & 0xFFFF0000u), s = b - __uint_as_float(v & 0xFFFF0000u);
        p.m[i] = pack_bf16(r, s);
        p.l[i] = pack_bf16(r - __uint_as_float(p.m[i] << 16), s - __uint_as_float(p.m[i] & 0xFFFF0000u));
    }
    if (most >= 0x7F800000u) {
        odd = true;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t u = __float_as_uint(i < 4 ? x[i] : y[i - 4]), low = i % 2 ? 0xFFFFu : 0xFFFF0000u;       // (low: of the other channel of the pair)
            if ((u & 0x7F800000u) != 0x7F800000u) continue;
            const uint32_t h = u & 0x7FFFFFu ? 0x7FC0u : u >> 16;
            p.h[i / 2] = (p.h[i / 2] & low) | (i % 2 ? h << 16 : h);
            p.m[i / 2] &= low;
            p.l[i / 2] &= low;
        }
    }
    return p;
}
__device__ __forceinline__ float whole(const Parts& p, int i) {    // channel i again
    const auto of = [&](uint32_t x) { return __uint_as_float(i % 2 ? x & 0xFFFF0000u : x << 16); };
    return of(p.h[i / 2]) + (of(p.m[i / 2]) + of(p.l[i / 2]));
}
template <> struct Many<false> {
    static constexpr int kBlocks = 1, kTiles = 2, kRow = 512;
    Parts x[8];
    bool odd;                          // of any lane's
    __device__ __forceinline__ void load(const char* row, int half) {
        f32x4a y[16];
#pragma unroll
        for (int s = 0; s < 8; ++s) y[2 * s] = ((const f32x4a*)row)[4 * s + 2 * half], y[2 * s + 1] = ((const f32x4a*)row)[4 * s + 2 * half + 1];
        bool mine = false;
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] = parts_of(y[2 * s], y[2 * s + 1], mine);
        odd = __any(mine);
    }
};

// Where a row R = (token, head of the group) lies, moved on by as many rows at a time without a division; units are the caller's.
struct Walk {
    uint32_t at;
    int i;
    __device__ __forceinline__ Walk(int R, const Divisor& group, uint32_t per_token, uint32_t per_head) {
        const int t = group.of(R);
        i = group.rest(R, t);
        at = t * per_token + i * per_head;
    }
    // heads: of the move beyond whole tokens; step: of all of it; wrap: from a token's end to the next one's start
    __device__ __forceinline__ void on(int heads, uint32_t step, uint32_t wrap, int group) {
        i += heads;
        at += step;
        const bool over = i >= group;
        i -= over ? group : 0;
        at += over ? wrap : 0;
    }
};

// The rows that keys j0 .. j1 are seen by, from the start of a stage on: its first one, and how many.
struct Span {
    int begin, stages;
};
__device__ __forceinline__ Span rows_that_see(const WeightsArgs& a, int length, int j0, int j1, int stage) {
    const Tokens t = tokens_that_see(length, a.c.m, j0, j1, a.c.window, a.c.sinks);
    const int begin = t.first * a.c.group / stage * stage, end = (t.last + 1) * a.c.group;
    return {begin, j0 <= j1 && begin < end ? (end - begin + stage - 1) / stage : 0};
}

// A head's products are shared out over `shares` workgroups by the cost of its tiles of keys, one after the other: their stages, and kTileCost for the keys and the masks at a tile's
// first ones.  Share s of n, no more than the total, has what lies in [total s / n, total (s + 1) / n).
constexpr int kTileCost = 6;
template <int KEYS, int STAGE>
struct Shares {
    const WeightsArgs& a;
    int length;
    __device__ __forceinline__ int stages(int tile) const {
        return tile < a.key_tiles ? rows_that_see(a, length, tile * KEYS, min(tile * KEYS + KEYS, length) - 1, STAGE).stages : 0;
    }
    static __device__ __forceinline__ int cost(int stages) { return stages > 0 ? stages + kTileCost : 0; }
    // the cost of the tiles below `tile`
    __device__ __forceinline__ int64_t below(int tile) const {
        int64_t sum = 0;
        for (int base = 0; base < tile; base += 64) {
            const int at = base + (int)(threadIdx.x & 63);
            sum += __builtin_amdgcn_readlane(up_to(at < tile ? cost(stages(at)) : 0), 63);
        }
        return sum;
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

// Stages from .. to - 1 of a tile of keys; `more`: the same workgroup has written this tile's sums before.
template <bool BF16>
__device__ __forceinline__ void tile_stages(const WeightsArgs& a, char (*Qs)[32768], float (*Ls)[Many<BF16>::kTiles * 32], int (*odd)[2], int g, int b, int head, int length, int key_tile, int begin,
                                            int stages, float* part, bool more) {
    typedef Many<BF16> M;
    constexpr int kKeys = M::kBlocks * 32, kTiles = M::kTiles, kStage = kTiles * 32;
    const WeightsCall& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int j0 = key_tile * (4 * kKeys);

    // Rows on their way into LDS: tiles of 32 rows, in columns of 64 bytes a row, pieces of 16 permuted by (row / 2) % 4.  bf16: a wave has a tile, in eight blocks of 16 rows' columns;
    // two stages of room.  fp32: a thread has 32 channels of a row, takes them apart and writes a column of each part, parts 16 KB apart; one stage of room, the next one's rows wait
    // in registers.
    const int piece = (lane & 3) ^ ((lane >> 3) & 3), my_row = BF16 ? wave * 32 + (lane >> 2) : tid >> 2;
    const uint32_t per_token = c.kv * c.group * M::kRow, over = per_token - c.group * M::kRow;
    const int first_token = a.by_group.of(begin), first_row = first_token * c.group;               // (offsets count from here)
    const int move_tokens = a.by_group.of(kStage), move_heads = a.by_group.rest(kStage, move_tokens);
    const char* queries = (const char*)uniform((int64_t)((const char*)c.Q + ((((int64_t)b * c.m + first_token) * c.kv + head) * c.group) * M::kRow));
    Walk low(begin - first_row + my_row, a.by_group, per_token, M::kRow), high(begin - first_row + my_row + 16, a.by_group, per_token, M::kRow);       // (bf16: the tile's halves)
    const float* lse_of_head = (const float*)uniform((int64_t)(c.lse + ((int64_t)b * c.kv + head) * c.group * c.m + first_token));
    Walk less_of(begin - first_row + tid % kStage, a.by_group, 1, c.m);
    float next_less = 0.f;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(&Qs[0][0]) + wave * 8192);
    f32x4a raw[BF16 ? 1 : 8];
    const auto ask = [&](int stage) ALWAYS_INLINE {
        const uint32_t within = BF16 ? piece * 16 : (tid & 3) * 128;
        uint32_t at[2] = {low.at + within, high.at + within}, l = less_of.at;
        if (begin + (stage + 1) * kStage > a.rows) {               // (what is behind the last row is not used)
            const int R = begin + stage * kStage;
            if (R + my_row >= a.rows) at[0] = within;
            if (R + my_row + 16 >= a.rows) at[1] = within;
            if (R + tid % kStage >= a.rows) l = 0;
        }
        if constexpr (BF16) {
            const uint32_t to = lds + (stage & 1) * 32768;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) dma16(to + h * 1024 + i * 2048, queries, at[h] + i * 64);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[i] = *(const f32x4a*)(queries + at[0] + i * 16);
        }
        next_less = lse_of_head[l];
        low.on(move_heads, move_tokens * per_token + move_heads * M::kRow, over, c.group);
        if (BF16) high.on(move_heads, move_tokens * per_token + move_heads * M::kRow, over, c.group);
        less_of.on(move_heads, move_tokens + move_heads * c.m, 1 - c.group * c.m, c.group);
    };
    const auto arrive = [&](int stage) ALWAYS_INLINE {
        if constexpr (!BF16) {
            if (tid == 0) odd[stage & 1][0] = 0;
            __syncthreads();                                       // (nobody reads the stage before any more)
            bool mine = false;
            char* to = Qs[0] + (my_row >> 5) * 8192 + (tid & 3) * 2048 + (my_row & 31) * 64;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Parts p = parts_of(raw[2 * i], raw[2 * i + 1], mine);
                const int of = (i ^ ((my_row >> 1) & 3)) << 4;
                *(u32x4a*)(to + of) = p.h;
                *(u32x4a*)(to + 16384 + of) = p.m;
                *(u32x4a*)(to + 32768 + of) = p.l;
            }
            if (mine) odd[stage & 1][0] = 1;
        }
        if (tid < kStage) {
            Ls[stage & 1][tid] = next_less == -INFINITY ? -INFINITY : -next_less * (1.f / kLn2);
            if constexpr (BF16) odd[stage & 1][wave] = __any(next_less == -INFINITY);
        }
        if constexpr (BF16) dma_wait();
        __syncthreads();
    };
    __syncthreads();                                               // (nobody reads the tile's before any more)
    if (stages > 0) ask(0);

    // This wave's keys; the stages of which its keys are seen at all, and those whose rows all see all of them.
    const int k0 = j0 + wave * kKeys, k1 = min(k0 + kKeys, length) - 1;
    M keys[M::kBlocks];
#pragma unroll
    for (int kb = 0; kb < M::kBlocks; ++kb) keys[kb].load((const char*)c.K + ((int64_t)g * c.stride + min(k0 + kb * 32 + col, length - 1)) * M::kRow, half);
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
    float sums[M::kBlocks * 16];
#pragma unroll
    for (int i = 0; i < M::kBlocks * 16; ++i) sums[i] = 0.f;
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    // A stage of which some rows do not see some of the wave's keys, or are none.
    const auto masked_stage = [&](int stage) ALWAYS_INLINE {
#pragma unroll 1
        for (int u = 0; u < kTiles; ++u) {
            const int R = begin + stage * kStage + u * 32 + col;
            const float less = Ls[stage & 1][u * 32 + col];
            // the keys that this lane's row sees, from k0 + 4 half on: up to `far`, but for those at `near` and below that are not below `first`
            const int at = R < a.rows && less != -INFINITY ? length - c.m + a.by_group.of(R) : -1, far = at - k0 - half * 4;
            uint64_t seen = far < 0 ? 0 : far >= 63 ? ~0ull : (2ull << far) - 1;
            if (c.window > 0) {
                const int64_t near = (int64_t)far - c.window, first = (int64_t)c.sinks - k0 - half * 4;
                seen &= (near < 0 ? ~0ull : near >= 63 ? 0ull : ~((2ull << near) - 1)) | (first <= 0 ? 0ull : first >= 64 ? ~0ull : (1ull << first) - 1);
            }
            if (!__any(seen != 0)) continue;
            const char* Qt = Qs[BF16 ? stage & 1 : 0] + u * 8192;
#pragma unroll
            for (int kb = 0; kb < M::kBlocks; ++kb) {
                f32x16a x;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = 0.f;
                if constexpr (BF16) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const u32x4a q = *(const u32x4a*)(Qt + k_at[i & 1] + (i >> 1) * 2048);
                        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, keys[kb].x[i]), __builtin_bit_cast(bf16x8a, q), x, 0, 0, 0);
                    }
                } else {
                    Parts q[2];
                    const auto read = [&](int i) ALWAYS_INLINE {
                        const char* from = Qt + k_at[i & 1] + (i >> 1) * 2048;
                        q[i & 1] = {*(const u32x4a*)from, *(const u32x4a*)(from + 16384), *(const u32x4a*)(from + 32768)};
                    };
                    read(0);
                    if (!keys[0].odd && odd[stage & 1][0] == 0) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (i < 7) read(i + 1);
                            const Parts &k = keys[0].x[i], &r = q[i & 1];
                            const auto add = [&](u32x4a y, u32x4a z) ALWAYS_INLINE {
                                x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, y), __builtin_bit_cast(bf16x8a, z), x, 0, 0, 0);
                            };
                            add(k.l, r.h), add(k.h, r.l), add(k.m, r.m), add(k.m, r.h), add(k.h, r.m), add(k.h, r.h);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (i < 7) read(i + 1);
                            Parts k = keys[0].x[i];
                            loaded(k.h), loaded(k.m), loaded(k.l);             // (put together here, not before the loop)
#pragma unroll
                            for (int e = 0; e < 8; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(whole(k, e), whole(q[i & 1], e), x, 0, 0, 0);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t keep = (int)((uint32_t)(seen >> (kb * 32)) << (31 - (i / 4 * 8 + i % 4))) >> 31;        // all bits, or none
                    sums[kb * 16 + i] += __uint_as_float(__float_as_uint(__builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less))) & keep);
                }
            }
        }
    };
    if (stages > 0) arrive(0);
    if constexpr (BF16)
#pragma unroll
        for (int kb = 0; kb < M::kBlocks; ++kb)
#pragma unroll
            for (int i = 0; i < 8; ++i) loaded(keys[kb].x[i]);
    // A row that gives nothing (lse -infinity) does so whatever its scores are, NaN and infinities among them: a stage that has one goes with masks (to look costs 3 us of a prompt of 8192
    // tokens' 290; with the next stage asked for between the look and the branch 2, but 31 us become 40 in fp32, by spills).
    const auto all_give = [&](int stage) ALWAYS_INLINE { return !BF16 || __builtin_amdgcn_readfirstlane(odd[stage & 1][0] | odd[stage & 1][1]) == 0; };
    int stage = 0;
#pragma unroll 1
    while (stage < stages) {                                       // stages with masks, whole ones, some with masks again
#pragma unroll 1
        for (; stage < stages && (stage < whole_from || stage >= whole_to || !all_give(stage)); ++stage) {
            if (stage + 1 < stages) ask(stage + 1);
            if (stage >= seen_from && stage < seen_to) masked_stage(stage);
            if (stage + 1 < stages) arrive(stage + 1);
        }
        if (stage >= stages) break;
        if constexpr (BF16) {
            // The scores of one tile wait for the next one's products, between which their exponentials go: two products, of either 32 keys, then two scores' of each.
            f32x16a s[2][2];
            float less[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 16; ++i) s[1][0][i] = s[1][1][i] = 0.f;
            u32x4a q[4];
            const auto read = [&](const char* Qt, int i) ALWAYS_INLINE { q[i & 3] = *(const u32x4a*)(Qt + k_at[i & 1] + (i >> 1) * 2048); };
            const auto tile = [&](int now, const char* Qt, const char* next) ALWAYS_INLINE {
                const f32x16a zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i < 6) read(Qt, i + 2);
                    else read(next, i - 6);
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) {
                        s[now][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, keys[kb].x[i]), __builtin_bit_cast(bf16x8a, q[i & 3]), i == 0 ? zero : s[now][kb], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int e = 2 * i; e < 2 * i + 2; ++e)
                            sums[kb * 16 + e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[now ^ 1][kb][e], a.scale_log2, less[now ^ 1]));
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
#pragma unroll 1
            for (; stage < whole_to && all_give(stage); ++stage) {
                if (stage + 1 < stages) ask(stage + 1);
                const char* Qt = Qs[stage & 1];
                read(Qt, 0);
                read(Qt, 1);
#pragma unroll 1
                for (int u = 0; u < kTiles; u += 2) {
                    less[0] = Ls[stage & 1][u * 32 + col];
                    tile(0, Qt, Qt + 8192);
                    less[1] = Ls[stage & 1][u * 32 + 32 + col];
                    tile(1, Qt + 8192, u + 2 < kTiles ? Qt + 16384 : Qt);
                    Qt += 16384;
                }
                if (stage + 1 < stages) arrive(stage + 1);
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[kb * 16 + i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[1][kb][i], a.scale_log2, less[1]));
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
    if (part) part[j - j0] = more ? part[j - j0] + sums[0] : sums[0];
    else add_to(c, g, j, sums[0], more ? 1.f : c.decay);
}

template <bool BF16>
__global__ __launch_bounds__(256, 2) void weights_many_kernel(WeightsArgs a) {
    constexpr int kKeys = Many<BF16>::kBlocks * 128, kStage = Many<BF16>::kTiles * 32;
    __shared__ __attribute__((aligned(16))) char Qs[2][32768];
    __shared__ float Ls[2][kStage];                                // -lse of a stage's rows, in units of log 2
    __shared__ int odd[2][2];                                      // of a stage: whether its rows hold an infinity or NaN (fp32), whether some of its halves' rows give nothing (bf16)
    const WeightsCall& c = a.c;
    // Neighbours in a head are neighbours in an XCD, whose caches then hold one head's queries.
    const int at = a.by_groups.of(blockIdx.x), g = a.by_groups.rest(blockIdx.x, at), b = a.by_kv.of(g), head = a.by_kv.rest(g, b), length = length_of(c, b);
    const auto run = [&](int tile, int from, int to, float* part) ALWAYS_INLINE {
        const Span span = rows_that_see(a, length, tile * kKeys, min(tile * kKeys + kKeys, length) - 1, kStage);
        for (int s = from; s == from || s < to; s += a.most)
            tile_stages<BF16>(a, Qs, Ls, odd, g, b, head, length, tile, span.begin + s * kStage, min(a.most, to - s), part, s > from);
    };
    if (a.shares == 0) {
        if (at * kKeys < length) run(at, 0, rows_that_see(a, length, at * kKeys, min(at * kKeys + kKeys, length) - 1, kStage).stages, nullptr);
        return;
    }
    const Shares<kKeys, kStage> shares{a, length};
    const int64_t total = shares.below(a.key_tiles), parts = min((int64_t)a.shares, total);
    if (at >= parts) return;
    const int64_t low = total * at / parts, high = total * (at + 1) / parts;
    int64_t before = 0;
    for (int base = 0; base < a.key_tiles && before < high; base += 64) {
        const int stages = shares.stages(base + (int)(threadIdx.x & 63)), sum = up_to(shares.cost(stages));
        const int64_t mine = before + sum - stages;                // where the tile's stages begin
        const int from = (int)min(max(low - mine, (int64_t)0), (int64_t)stages), to = (int)min(max(high - mine, (int64_t)0), (int64_t)stages);
        before += __builtin_amdgcn_readlane(sum, 63);
        for (uint64_t some = __ballot(from < to); some; some &= some - 1) {
            const int l = __builtin_ctzll(some), tile = base + l;
            run(tile, __builtin_amdgcn_readlane(from, l), __builtin_amdgcn_readlane(to, l), a.part + ((int64_t)g * (a.shares + a.key_tiles) + at + tile) * kKeys);
        }
    }
}

// ---- up to 128 rows, bf16: they lie in LDS once for all, and each wave goes over blocks of 32 keys of its own, the next one on its way (two on their way: 19.3 us where one takes 18.4).
__global__ __launch_bounds__(256, 3) void weights_some_kernel(WeightsArgs a) {
    __shared__ __attribute__((aligned(16))) char Qs[32768];
    __shared__ float less_of[128];
    __shared__ int place_of[128];
    const WeightsCall& c = a.c;
    const int head = blockIdx.x % c.kv, share = blockIdx.x / c.kv % a.shares, b = blockIdx.x / c.kv / a.shares, g = b * c.kv + head;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int length = length_of(c, b), blocks = (length + 31) / 32, tiles = (a.rows + 31) / 32;
    const int first = share * 4, step = a.shares * 4;              // (neighbours' blocks are neighbours, so that what a window hides is shared out evenly)
    if (first >= blocks) return;
    const char* queries = (const char*)uniform((int64_t)((const char*)c.Q + ((int64_t)b * c.m * c.kv + head) * c.group * 256));
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(&Qs[0]) + wave * 8192);
#pragma unroll
    for (int h = 0; h < 2; ++h) {                                  // (columns of 64 bytes a row, as in tile_stages)
        const int R = min(wave * 32 + h * 16 + (lane >> 2), a.rows - 1), token = a.by_group.of(R);
        const uint32_t at = (uint32_t)(token * c.kv * c.group + a.by_group.rest(R, token)) * 256 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) dma16(lds + h * 1024 + i * 2048, queries, at + i * 64);
    }
    const char* keys = (const char*)c.K + (int64_t)g * c.stride * 256;
    Many<true> next;
    const auto ask = [&](int block) ALWAYS_INLINE {
        if ((block < blocks) & any_sees(c, length, block * 32, block * 32 + 31)) next.load(keys + (int64_t)min(block * 32 + col, length - 1) * 256, half);
    };
    ask(first + wave);
    if (tid < 128) {                                               // of a row -lse in units of log 2, and its position (below all where it gives nothing)
        const int R = min(tid, a.rows - 1), token = a.by_group.of(R);
        const float lse = c.lse[(((int64_t)b * c.kv + head) * c.group + a.by_group.rest(R, token)) * c.m + token];
        less_of[tid] = -lse * (1.f / kLn2);
        place_of[tid] = tid < a.rows && lse != -INFINITY ? length - c.m + token : -1;
    }
    dma_wait();
    __syncthreads();
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    const int mine = (col & 15) / 4 * 8 + col % 4 + half * 4;      // the key of a block whose sum comes to this lane
    float* mass = c.mass + (int64_t)g * c.mass_stride;
#pragma unroll 1
    for (int block = first + wave; block < blocks; block += step) {
        const int k0 = block * 32, j = k0 + mine;
        const Many<true> key = next;
        ask(block + step);
        const float old = mass[min(j, length - 1)];
        float sums[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[i] = 0.f;
        const int seen_tiles = any_sees(c, length, k0, k0 + 31) ? tiles : 0;
#pragma unroll 1
        for (int u = 0; u < seen_tiles; ++u) {                     // (not unrolled: a launch of few blocks pays for the code that it fetches)
            const char* Qt = Qs + u * 8192;
            const float less = less_of[u * 32 + col];
            const int p = place_of[u * 32 + col];
            f32x16a x;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const u32x4a q = *(const u32x4a*)(Qt + k_at[i & 1] + (i >> 1) * 2048);
                x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, key.x[i]), __builtin_bit_cast(bf16x8a, q), x, 0, 0, 0);
            }
            if (__all(k0 + 31 <= p && (c.window == 0 || k0 + 31 < c.sinks || p - k0 < c.window))) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less));
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, less));
                    sums[i] += sees(p, k0 + i / 4 * 8 + i % 4 + half * 4, c.window, c.sinks) ? w : 0.f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[i] += __shfl_xor(sums[i], 16);
        spread<8>(sums, col);
        if (j < length && col < 16) mass[j] = c.decay == 0.f ? sums[0] : __builtin_fmaf(c.decay, old, sums[0]);
    }
}

// Adds up the shares of a key's tile, in order; a wave's keys are of one tile.
template <bool BF16>
__global__ __launch_bounds__(256) void weights_join_kernel(WeightsArgs a) {
    constexpr int kKeys = Many<BF16>::kBlocks * 128, kStage = Many<BF16>::kTiles * 32;
    const WeightsCall& c = a.c;
    const int block = a.by_groups.of(blockIdx.x), g = a.by_groups.rest(blockIdx.x, block), j = block * 256 + threadIdx.x, length = length_of(c, a.by_kv.of(g));
    const int tile = __builtin_amdgcn_readfirstlane(j / kKeys);
    const Shares<kKeys, kStage> shares{a, length};
    const int stages = shares.stages(tile);
    float sum = 0.f;
    if (stages > 0) {
        // the share of position x is the largest s with total s / parts <= x
        const int64_t total = shares.below(a.key_tiles), first = shares.below(tile) + kTileCost, parts = min((int64_t)a.shares, total);
        const int from = (int)(((first + 1) * parts - 1) / total), to = (int)(((first + stages) * parts - 1) / total);
        const float* part = a.part + ((int64_t)g * (a.shares + a.key_tiles) + tile) * kKeys + j % kKeys;
        for (int s = from; s <= to && j < length; s += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = part[(int64_t)min(s + e, to) * kKeys];
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += s + e <= to ? x[e] : 0.f;
        }
    }
    if (j < length) add_to(c, g, j, sum, c.decay);
}

}  // namespace

hipError_t launch_weights(const curdkv_ctx* ctx, const WeightsCall& call, hipStream_t stream) {
    const bool bf16 = call.dtype == CURDKV_DTYPE_BF16;
    WeightsArgs a{call, call.scale * (1.f / kLn2), (int)(call.count * call.kv), call.m * call.group, 0, 0, 0, nullptr, Divisor(call.count * call.kv), Divisor(call.kv), Divisor(call.group)};
    const bool past = (int64_t)a.groups * call.n * (bf16 ? 256 : 512) > kPastCaches;
    if (a.rows <= 32 && (past || !bf16 || (a.rows <= 16 && (int64_t)a.groups * call.n <= 512 * (int64_t)ctx->num_cu))) {
        const int64_t steps = (call.n + 63) / 64, waves = 16 * (int64_t)ctx->num_cu;
        const int64_t each = std::max<int64_t>(1, std::min<int64_t>(4, a.groups * steps / waves));
        a.shares = (int)((steps + 4 * each - 1) / (4 * each));
        const auto launch = [&](auto kernel) { kernel<<<(unsigned)((int64_t)a.groups * a.shares), 256, 0, stream>>>(a); };
        if (bf16 && a.rows <= 16) past ? launch(weights_few_kernel<true, 1, true>) : launch(weights_few_kernel<true, 1, false>);
        else if (bf16) launch(weights_few_kernel<true, 2, true>);
        else if (a.rows <= 16) past ? launch(weights_few_kernel<false, 1, true>) : launch(weights_few_kernel<false, 1, false>);
        else past ? launch(weights_few_kernel<false, 2, true>) : launch(weights_few_kernel<false, 2, false>);
        return hipGetLastError();
    }
    if (bf16 && a.rows <= 128) {                                   // two workgroups a unit, as far as each of their waves has a block of keys (three: 19.2 us where two take 18.6)
        const int64_t blocks = (call.n + 31) / 32;
        a.shares = (int)std::max<int64_t>(1, std::min<int64_t>((blocks + 3) / 4, 2 * (int64_t)ctx->num_cu / a.groups));
        weights_some_kernel<<<(unsigned)((int64_t)a.groups * a.shares), 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    const int keys = bf16 ? 256 : 128, stage = bf16 ? 128 : 64;
    a.key_tiles = (call.n + keys - 1) / keys;
    a.most = (int)(((int64_t)1 << 31) / (call.kv * (bf16 ? 256 : 512)) / stage);
    // Two workgroups a unit, each with an equal share of a head's products, where tiles of keys would leave units idle at the end; their sums lie in scratch, as far as there is any.
    // (1021 tokens over 1021: 22 us so, 85 by tiles; 2000 over 2000: 45 and 146.  Up to four stages of rows there is little to share: 100 tokens over 8000 24.7 so, 17.3 by tiles.)
    const int64_t tiles = (int64_t)a.groups * a.key_tiles, room = call.scratch ? (call.scratch_bytes - kScratchCounters) / (a.groups * (int64_t)keys * 4) - a.key_tiles : 0;
    const int64_t shares = std::min(std::min<int64_t>(2 * (int64_t)ctx->num_cu / a.groups, room), std::max<int64_t>(1, (int64_t)((a.rows + stage - 1) / stage) * a.key_tiles));
    a.shares = tiles < 2 * (int64_t)ctx->num_cu && a.rows > 4 * stage && shares > 1 ? (int)shares : 0;
    a.part = (float*)((char*)call.scratch + kScratchCounters);
    const auto launch = [&](auto kernel, int64_t n) { kernel<<<(unsigned)n, 256, 0, stream>>>(a); };
    const int64_t blocks = a.shares ? (int64_t)a.groups * a.shares : tiles;
    bf16 ? launch(weights_many_kernel<true>, blocks) : launch(weights_many_kernel<false>, blocks);
    if (a.shares) {
        const int64_t joins = (int64_t)a.groups * ((call.n + 255) / 256);
        bf16 ? launch(weights_join_kernel<true>, joins) : launch(weights_join_kernel<false>, joins);
    }
    return hipGetLastError();
}

}  // namespace curdkv
