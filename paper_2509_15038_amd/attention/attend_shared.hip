// Attention of many sequences over the kept rows that they share, and over their own tails: of two sets of keys with (M1, L1, o1) and (M2, L2, o2), o un-normalised,
// the whole has M = max, L = L1 2^(M1-M) + L2 2^(M2-M) and o likewise (scores in units of log 2).  So the rows R of all of a prefix's
// sequences (R = (sequence, token, head)) stand side by side over its kept rows, which are read once for a tile of up to 256 of them, each
// sequence's own over its tail, and a second kernel joins what they found.
//
// One launch: workgroups of tails (a sequence's KV head, 32 rows R, by four waves that take tiles of 32 keys in turn and are joined in LDS, or by one), then those of kept rows, which share out
// all heads' tiles evenly, whatever the heads' lengths.  S^T = K Q^T and O^T = V^T P^T by mfma_f32_32x32x16_bf16, operands and layout of the tiles in LDS as in attend_prompt.hip: columns of 64 bytes a
// row, V read transposed, P from the registers that S^T leaves it in.  Four (eight) waves have 32 of 128 (256) rows each and all of a tile's 64 keys.  Rows in 4 bits are expanded on their way
// into LDS, exactly.  fp32: mfma_f32_32x32x2, operands straight from memory.
// Weights are rounded to bf16 for their product with V (by up to 2^-8 of themselves, as the values have been and the result will be: 0.0021 to 0.0023 of the result in all, root mean square, 0.0016
// to 0.0017 without); sums are of what was not rounded.
//
// Bound by: over long prefixes the products, for 42 % of the clocks, which wait for tiles and exponentials, and, for a fifth, the power that lowers the clock to 1.9 to 2.1 GHz (64 sequences
// over 131072 kept rows of 8 heads, 137 GFLOP, 557 MB, 177 us: 780 TFLOP/s; with zeros for numbers 148); in 4 bits the expansion, which every 128 rows take anew, by the waves that have the
// products too (4 prompts of 13107 kept rows, 16 answers to each with up to 513 tokens, 124 MB, 59 us, of which the tails' 83 MB 13); over short ones the chain of two
// launches, a few tiles that each wait for all copies asked for, and the join (16 answers over 3276 rows, 21 MB, 18.4 us).  fp32: 16 answers over 13107 rows 53 to 60 us, of which the products of
// 32 bits 25, and 39 of one answer, whose tiles of 32 rows are filled to an eighth.
// Tails are not cut into parts: one of 2048 tokens takes the whole 22 us, of 32768 213 (curdkv_attend_kept 14 and 34), in fp32 81 and 1125 (21 and 64).
#include <algorithm>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

typedef short s16x4a __attribute__((ext_vector_type(4)));

constexpr float kLoose = 8.f;          // a reference point may lie so far below the maximum (weights up to 2^8)
constexpr int kTile = 32;              // rows R of a wave

struct SharedArgs {
    AttendCall c;
    float scale_log2;
    int share;
    // this launch's slice: sequences s0 .. s0 + ns - 1 of prefixes b0 .. b0 + nb - 1, tokens t0 .. t0 + nt - 1
    int b0, nb, s0, ns, t0, nt;
    int rows, tile_rows, tiles;        // of a prefix's KV head: ns * nt * group, and tiles of tile_rows of them
    int slot_rows;                     // of a part: a tile's, where there is but one no more than there are
    int shares;                        // workgroups that share out the kept rows
    int tail_tiles;                    // tiles of 32 of a sequence's nt * group rows
    int tail_waves;                    // of a tail: four, or, where there are many tails, one
    int64_t tails, tail_blocks;
    // un-normalised partial results of 128 floats a row, and their reference points and sums (sum 0: nothing seen, o not written): of share s and item i, (head, tile), at s + i, which
    // no other pair has, [shares + items][slot_rows], then of the tails [nb * kv][rows]
    float* part_o;
    f32x2a* part_ml;
    int32_t* part_of_item;             // the first and the last share that have tiles of an item (of a head without kept rows: not written)
    int64_t tail_at;                   // rows before the tails'
    Divisor by_group, by_per, by_kv, by_tail_tiles, by_ns, by_quads;       // by_per: by a sequence's rows, nt * group; by_quads: by fours of a head's rows
};

// Rows R of a workgroup, first .. end - 1 of a head's (or of one sequence's), and where row R's partial result lies, at + R.
struct Rows {
    int64_t at;
    int first, end;
};

__device__ __forceinline__ f32x16a product(u32x4a x, u32x4a y, f32x16a z) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, x), __builtin_bit_cast(bf16x8a, y), z, 0, 0, 0);
}
__device__ __forceinline__ u32x2 read_transposed(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4a*)p));
}
__device__ __forceinline__ float unit_of(uint32_t scale) { return __uint_as_float(scale << 23); }      // (the conversions take the exponent alone: 0 is 2^-127, 255 NaN)
template <int SEL>
__device__ __forceinline__ uint32_t two_bf16(uint32_t codes, float unit) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, SEL));
}
template <int SEL>
__device__ __forceinline__ f32x2a two_f32(uint32_t codes, float unit) {
    return __builtin_bit_cast(f32x2a, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, SEL));
}
__device__ __forceinline__ u32x4a eight_bf16(uint32_t codes, float unit) {
    return (u32x4a){two_bf16<0>(codes, unit), two_bf16<1>(codes, unit), two_bf16<2>(codes, unit), two_bf16<3>(codes, unit)};
}

// The global row of row R of prefix bi's head (of the slice), and its token.
__device__ __forceinline__ int64_t query_row(const SharedArgs& a, int bi, int head, int R, int* token) {
    const int s = a.by_per.of(R), in = a.by_per.rest(R, s), t = a.by_group.of(in);
    *token = a.t0 + t;
    return ((((int64_t)(a.b0 + bi) * a.share + a.s0 + s) * a.c.m + a.t0 + t) * a.c.kv + head) * a.c.group + a.by_group.rest(in, t);
}

// The kept rows of head g of the slice: where they begin, and how many there are.
struct Kept {
    int64_t at;
    int count;
};
__device__ __forceinline__ Kept kept_rows(const SharedArgs& a, int g) {
    const int64_t* offsets = a.c.offsets + (int64_t)a.b0 * a.c.kv + g;
    const int64_t begin = min(max(offsets[0], (int64_t)0), a.c.total);
    return {begin, (int)(min(max(offsets[1], begin), a.c.total) - begin)};
}
// The kept rows' tiles of 64 keys are shared out by their cost, head after head and within a head row tile after row tile: a tile each, and kItemCost for every (head, row tile).
// Shares are equal, the first of them longer by one, and no more than the total.
constexpr int kItemCost = 2;
__device__ __forceinline__ int cost_of(int count) { return count > 0 ? (count + 63) / 64 + kItemCost : 0; }
// A wave's 32 rows R over tiles of KEYS keys in LDS.
struct Wave {
    u32x4a q[8];
    f32x16a o[4];
    float ref, sum;
    __device__ __forceinline__ void begin(const char* row, int half) {
#pragma unroll
        for (int s = 0; s < 8; ++s) q[s] = ((const u32x4a*)row)[2 * s + half];
        ref = kNoScore, sum = 0.f;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    }
    // where step i's operand lies in its column, k_at being step 0's
    template <int STRIDE>
    static __device__ __forceinline__ int key_at(int k_at, int i) {
        return k_at ^ ((2 * (i & 1) ^ (STRIDE == 4096 ? i >> 1 : 0)) << 4);
    }
    // KB blocks of 32 keys, columns STRIDE bytes apart
    template <int KB, int STRIDE>
    __device__ __forceinline__ void scores(const char* Kt, int col, int half, f32x16a (&x)[KB]) const {
        const int k_at = col * 64 + ((half ^ ((col >> 1) & 3)) << 4);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kb][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[kb] = product(*(const u32x4a*)(Kt + key_at<STRIDE>(k_at, i) + (i >> 1) * STRIDE + kb * 2048), q[i], x[kb]);
        }
    }
    template <int KB>
    __device__ __forceinline__ float top_of(const f32x16a (&x)[KB], float scale_log2) const {
        float top = x[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
        return halves_max(top) * scale_log2;
    }
    // the reference point moves where it lies too far below
    __device__ __forceinline__ void raise(float top) {
        if (__any(top > ref + kLoose)) {
            const float next = top > ref + kLoose ? top : ref, keep = next == ref ? 1.f : __builtin_amdgcn_exp2f(ref - next);
            sum *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db) o[db] *= keep;
            ref = next;
        }
    }
    // the weights of scores i and i + 1, a pair of bf16
    template <int KB>
    __device__ __forceinline__ uint32_t weigh(const f32x16a (&x)[KB], int i, float scale_log2) {
        const float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 4][i & 15], scale_log2, -ref));
        const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 4][(i & 15) + 1], scale_log2, -ref));
        sum += u + v;
        return pack_bf16(u, v);
    }
    template <int STRIDE>
    static __device__ __forceinline__ u32x4a value(const char* Vt, int v_at, int u, int db) {
        const char* p = Vt + (STRIDE == 4096 ? v_at ^ (db << 4) : v_at) + db * STRIDE + u * 1024;
        const u32x2 x = read_transposed(p), y = read_transposed(p + 512);
        return (u32x4a){x.x, x.y, y.x, y.y};
    }
    template <int KB, int STRIDE, bool FINITE>     // !FINITE: zeros in the place of infinities and NaN
    __device__ __forceinline__ void values(const char* Vt, int v_at, const uint32_t (&pb)[KB * 8]) {
#pragma unroll
        for (int u = 0; u < KB * 2; ++u)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                u32x4a w = value<STRIDE>(Vt, v_at, u, db);
                if (!FINITE)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((w[e] & 0x7F80u) == 0x7F80u) w[e] &= 0xFFFF0000u;
                        if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] &= 0x0000FFFFu;
                    }
                o[db] = product(w, (u32x4a){pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]}, o[db]);
            }
    }
};
// Scores of keys beyond `far` (counted from the half's first) are -infinity.
template <int KB>
__device__ __forceinline__ void hide(f32x16a (&s)[KB], int far) {
#pragma unroll
    for (int i = 0; i < KB * 16; ++i) s[i >> 4][i & 15] = (i >> 4) * 32 + (i & 15) / 4 * 8 + i % 4 <= far ? s[i >> 4][i & 15] : -INFINITY;
}

// Tiles of 32 or 64 keys in LDS: four columns of 64 bytes a row, K's pieces of 16 bytes permuted by (row / 2) % 4, and in tiles of 64 keys all by the column: four lanes that store a row
// in 4 bits have a column each, and would meet the same banks (16 answers over 131072 rows: 86 us without, 79 with; bf16, which DMA writes in whole lines, 113 either way).
__device__ __forceinline__ int permuted(int piece, int row, int column, bool keys, int keys_of_tile) {
    return piece ^ (keys_of_tile == 64 ? column : 0) ^ (keys ? (row >> 1) & 3 : 0);
}
// 1 KB blocks of 16 rows' columns, block first .. first + COUNT - 1 of a tile, straight into LDS.
template <int KEYS, int COUNT>
__device__ __forceinline__ void fetch_bf16(uint32_t lds, const char* rows, int count, bool keys, int first, int lane) {
    rows = (const char*)uniform((int64_t)rows);
    lds = __builtin_amdgcn_readfirstlane(lds);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int block = first + i, column = block / (KEYS / 16), row = block % (KEYS / 16) * 16 + (lane >> 2);
        dma16(lds + block * 1024, rows, min(row, count - 1) * 256 + column * 64 + (permuted(lane & 3, row, column, keys, KEYS) << 4));
    }
}
// Rows in 4 bits: a lane's share of a tile of 64 keys, a column of one row in 16 bytes of codes, and its scale.
struct Codes {
    u32x4a codes;
    uint32_t scale;
    __device__ __forceinline__ void load(const uint8_t* rows, const uint8_t* scales, int64_t row, int column) {
        codes = *(const u32x4a*)(rows + row * 64 + column * 16);
        scale = scales[row * 4 + column];
    }
    __device__ __forceinline__ void store(char* tile, int row, int column, bool keys) const {
#pragma unroll
        for (int p = 0; p < 4; ++p) *(u32x4a*)(tile + (uint32_t)(column * 4096 + row * 64 + (permuted(p, row, column, keys, 64) << 4))) = eight_bf16(codes[p], unit_of(scale));
    }
};

// Zeros in rows count .. KEYS - 1 of a tile of V, by LANES threads.
template <int KEYS, int LANES>
__device__ __forceinline__ void clear_beyond(char* tile, int count, int thread) {
    for (int i = count * 16 + thread; i < KEYS * 16; i += LANES) *(u32x4a*)(tile + (i & 3) * (KEYS * 64) + (i >> 4) * 64 + (i >> 2 & 3) * 16) = (u32x4a){0, 0, 0, 0};
}

// A partial result of 32 rows R: O^T's lanes (column R, channels 32 db + 8 i + 4 half ..) to rows of 128 floats.
__device__ __forceinline__ void store_part(const Wave& w, float* to, int half) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4a*)(to + db * 32 + i * 8 + half * 4) = (f32x4a){w.o[db][4 * i], w.o[db][4 * i + 1], w.o[db][4 * i + 2], w.o[db][4 * i + 3]};
}

// That of a wave of its own.
__device__ __forceinline__ void store_wave(const SharedArgs& a, const Wave& w, const Rows& r, int col, int half) {
    const float sum = halves_sum(w.sum);
    if (r.first + col >= r.end) return;
    if (half == 0) a.part_ml[r.at + r.first + col] = (f32x2a){w.ref, sum};
    if (sum != 0.f) store_part(w, a.part_o + (r.at + r.first + col) * 128, half);
}

// The parts of four waves (threads tid of them) over the same 32 rows R, through 16 KB of LDS each.
__device__ __forceinline__ void join_waves(Wave& w, int tid, char* lds, f32x2a (*ml)[kTile], float* part_o, f32x2a* part_ml, const Rows& r) {
    const int wave = tid >> 6, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const float sum = halves_sum(w.sum);
    __syncthreads();                   // (nobody reads tiles any more)
    if (half == 0) ml[wave][col] = (f32x2a){w.ref, sum};
    __syncthreads();
    const float ref = fmaxf(fmaxf(ml[0][col].x, ml[1][col].x), fmaxf(ml[2][col].x, ml[3][col].x));
    // (16-byte pieces permuted by the row, so that the rows of a store meet different banks)
    const float scale = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(w.ref - ref);
    float* to = (float*)lds + (wave * kTile + col) * 128;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4a*)(to + ((db * 8 + i * 2 + half) ^ (col & 7)) * 4) =
                (f32x4a){w.o[db][4 * i] * scale, w.o[db][4 * i + 1] * scale, w.o[db][4 * i + 2] * scale, w.o[db][4 * i + 3] * scale};
    __syncthreads();
    const int row = tid >> 3, R = r.first + row;
    if (R >= r.end) return;
    const float m = fmaxf(fmaxf(ml[0][row].x, ml[1][row].x), fmaxf(ml[2][row].x, ml[3][row].x));
    float l = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) l += ml[k][row].y == 0.f ? 0.f : ml[k][row].y * __builtin_amdgcn_exp2f(ml[k][row].x - m);
    if ((tid & 7) == 0) part_ml[r.at + R] = (f32x2a){m, l};
    if (l == 0.f) return;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int piece = (tid & 7) + p * 8;
        f32x4a x = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) x += *(const f32x4a*)((const float*)lds + (k * kTile + row) * 128 + (piece ^ (row & 7)) * 4);
        *(f32x4a*)(part_o + (r.at + R) * 128 + piece * 4) = x;
    }
}

// Infinities and NaN among a tile's values must not meet the zero weights of rows that do not see them: key j of 32 is seen where j <= far, of this half.  One wave.
__device__ __forceinline__ void hidden_values(Wave& w, const char* Vt, int v_at, const uint32_t (&pb)[8], int far, int half, int lane) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32x4a x = *(const u32x4a*)(Vt + i * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7F80u) == 0x7F80u || (x[e] & 0x7F800000u) == 0x7F800000u;
    }
    if (!__any(bad)) {
        w.values<1, 2048, true>(Vt, v_at, pb);
        return;
    }
    w.values<1, 2048, false>(Vt, v_at, pb);
    for (int key = 0; key < 32; ++key) {
        if (key - half * 4 > far) break;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x2 v = *(const u32x2*)(Vt + db * 2048 + key * 64 + i * 16 + half * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t x = e % 2 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16;
                    if ((x & 0x7F800000u) == 0x7F800000u) w.o[db][4 * i + e] += __uint_as_float(x);
                }
            }
    }
}

template <int LEFT>
__device__ __forceinline__ void dma_wait_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(LEFT) : "memory"); }      // all but the last LEFT
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A tail's 32 rows R, by WAVES waves, four or one (threads tid of them), each over tiles of 32 keys of its own, of which the next one's keys are on their way while the weights are made, and its values
// while they are.  Row R's token stands at p, the first row's at p_low.
template <int WAVES>
__device__ __forceinline__ void tail_rows(const SharedArgs& a, int tid, char* lds, uint32_t lds_at, f32x2a (*ml)[kTile], const char* K, const char* V, int end, int p, int p_low,
                                          const char* row, const Rows& r) {
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int v_at = (4 * half + l16 / 4) * 64 + (lane >> 4 & 1) * 32 + (l16 & 3) * 8;
    char *Kt = lds + wave * 16384, *Vt = Kt + 8192;
    const uint32_t k_lds = lds_at + wave * 16384, v_lds = k_lds + 8192;
    Wave w;
    const int tiles = (end + 31) / 32, last = min(p, end - 1);
    const auto count_of = [&](int tile) ALWAYS_INLINE { return min(32, end - tile * 32); };
    const auto ask_k = [&](int tile) ALWAYS_INLINE { fetch_bf16<32, 8>(k_lds, K + (int64_t)tile * 8192, count_of(tile), true, 0, lane); };
    const auto ask_v = [&](int tile) ALWAYS_INLINE { fetch_bf16<32, 8>(v_lds, V + (int64_t)tile * 8192, count_of(tile), false, 0, lane); };
    if (wave < tiles) {
        ask_k(wave);
        ask_v(wave);
    }
    w.begin(row, half);
#pragma unroll
    for (int i = 0; i < 8; ++i) loaded(w.q[i]);
    for (int tile = wave; tile < tiles; tile += WAVES) {
        const int j0 = tile * 32, count = count_of(tile);
        const bool more = tile + WAVES < tiles, hidden = count < 32 || j0 + 31 > p_low;
        dma_wait_but<8>();
        f32x16a s[1];
        uint32_t pb[8];
        w.scores<1, 2048>(Kt, col, half, s);
        lds_wait();
        if (more) ask_k(tile + WAVES);
        if (hidden) hide<1>(s, last - j0 - half * 4);
        w.raise(w.top_of<1>(s, a.scale_log2));
#pragma unroll
        for (int i = 0; i < 16; i += 2) pb[i / 2] = w.weigh<1>(s, i, a.scale_log2);
        if (more) dma_wait_but<8>();
        else dma_wait();
        if (count < 32) clear_beyond<32, 64>(Vt, count, lane);
        if (hidden) hidden_values(w, Vt, v_at, pb, last - j0 - half * 4, half, lane);
        else w.values<1, 2048, true>(Vt, v_at, pb);
        lds_wait();
        if (more) ask_v(tile + WAVES);
    }
    if constexpr (WAVES == 4) join_waves(w, tid, lds, ml, a.part_o, a.part_ml, r);
    else store_wave(a, w, r, col, half);
}

// 32 SETS rows R, 32 a wave, tiles of 64 keys for all.  The next tile's products go with this one's exponentials between them,
// this one's products with V with the next one's maximum: K is a tile ahead of V.  Rows in 4 bits wait in registers for a tile (two and three tiles were slower: spills).
template <bool MX, int SETS>
__device__ __forceinline__ void kept_rows_of(const SharedArgs& a, char* lds, uint32_t lds_at, const void* K, const void* V, const uint8_t* K_scales, const uint8_t* V_scales,
                                          int begin, int end, const char* row, const Rows& r) {
    constexpr int KB = 2, W = SETS;                                // blocks of 32 keys; waves
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int v_at = (4 * half + l16 / 4) * 64 + (lane >> 4 & 1) * 32 + (l16 & 3) * 8;
    const bool works = r.first + wave * kTile < r.end;      // (a wave without rows helps with the tiles)
    Wave w;
    const int tiles = (end - begin + 63) / 64;
    const auto count_of = [&](int tile) ALWAYS_INLINE { return min(64, end - begin - tile * 64); };
    // bf16: K or V of a tile on its way into LDS
    const auto fetch = [&](bool keys, int tile) ALWAYS_INLINE {
        if constexpr (!MX)
            fetch_bf16<64, 16 / W>(lds_at + (tile & 1) * 16384 + (keys ? 0 : 32768), (const char*)(keys ? K : V) + (int64_t)(begin + tile * 64) * 256, count_of(tile), keys,
                                   wave * (16 / W), lane);
    };
    // 4 bits: a thread's 32 channels of a row of K, and of V (of eight waves, four take K and four V), into registers and from there into LDS
    Codes codes[W == 8 ? 1 : 2];
    const int my_row = (tid & 255) >> 2, column = tid & 3;
    const auto load = [&](Codes& x, bool keys, int tile) ALWAYS_INLINE {
        const int t = min(tile, tiles - 1);
        const int64_t at = begin + t * 64 + min(my_row, count_of(t) - 1);
        x.load((const uint8_t*)(keys ? K : V), keys ? K_scales : V_scales, at, column);
    };
    const auto store = [&](const Codes& x, bool keys, int tile) ALWAYS_INLINE {
        if (tile < tiles) x.store(lds + (tile & 1) * 16384 + (keys ? 0 : 32768), my_row, column, keys);
    };
    const auto ask_both = [&](int tile) ALWAYS_INLINE {            // K of tile + 1, V of tile
        if constexpr (MX && W == 8) {
            load(codes[0], wave < 4, wave < 4 ? tile + 1 : tile);
        } else if constexpr (MX) {
            load(codes[0], true, tile + 1);
            load(codes[1], false, tile);
        }
    };
    const auto store_both = [&](int tile) ALWAYS_INLINE {
        if constexpr (MX && W == 8) {
            store(codes[0], wave < 4, wave < 4 ? tile + 1 : tile);
        } else if constexpr (MX) {
            store(codes[0], true, tile + 1);
            store(codes[1], false, tile);
        }
    };
    const auto arrive = [&](int values) ALWAYS_INLINE {            // values: the tile whose V is among what comes
        if constexpr (!MX) dma_wait();
        if (values < tiles && count_of(values) < 64) {
            __syncthreads();
            clear_beyond<64, W * 64>(lds + (values & 1) * 16384 + 32768, count_of(values), tid);
        }
        __syncthreads();
    };
    const auto keys_of = [&](int tile) ALWAYS_INLINE { return lds + (tile & 1) * 16384; };
    const auto values_of = [&](int tile) ALWAYS_INLINE { return lds + (tile & 1) * 16384 + 32768; };
    const auto mask = [&](f32x16a (&s)[KB], int tile) ALWAYS_INLINE {
        if (count_of(tile) < 64) hide<KB>(s, count_of(tile) - 1 - half * 4);
    };
    __syncthreads();                   // (nobody reads the item's before any more)
    // (begin < end)
    {
        if constexpr (MX) {
            Codes k;
            if (W == 4 || wave < 4) load(k, true, 0);
            ask_both(0);
            if (W == 4 || wave < 4) store(k, true, 0);
            store_both(0);
            ask_both(1);
        } else {
            fetch(true, 0);
            fetch(false, 0);
            if (tiles > 1) fetch(true, 1);
        }
        w.begin(row, half);
        arrive(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) loaded(w.q[i]);
        f32x16a s[KB];
        w.scores<KB, 4096>(keys_of(0), col, half, s);
        mask(s, 0);
        float top = w.top_of<KB>(s, a.scale_log2);
        __syncthreads();               // (K of tile 0 is read)
        const int k_at = col * 64 + ((half ^ ((col >> 1) & 3)) << 4);
        const auto step = [&](int tile) ALWAYS_INLINE {            // (with it come K of tile + 2 and V of tile + 1)
            if constexpr (!MX) {
                if (tile + 2 < tiles) fetch(true, tile + 2);
                fetch(false, tile + 1);
            }
            if (works) {
                w.raise(top);
                const char *Kt = keys_of(tile + 1), *Vt = values_of(tile);
                f32x16a next[KB];
                uint32_t pb[KB * 8];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) next[kb][i] = 0.f;
                u32x4a kk[2][KB];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) kk[0][kb] = *(const u32x4a*)(Kt + k_at + kb * 2048);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i < 7)
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) kk[(i + 1) & 1][kb] = *(const u32x4a*)(Kt + Wave::key_at<4096>(k_at, i + 1) + ((i + 1) >> 1) * 4096 + kb * 2048);
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) next[kb] = product(kk[i & 1][kb], w.q[i], next[kb]);
#pragma unroll
                    for (int j = 0; j < 2 * KB; j += 2) pb[(i * 2 * KB + j) / 2] = w.weigh<KB>(s, i * 2 * KB + j, a.scale_log2);
                    __builtin_amdgcn_sched_barrier(0);
                }
                u32x4a vv[2][4];
#pragma unroll
                for (int db = 0; db < 4; ++db) vv[0][db] = Wave::value<4096>(Vt, v_at, 0, db);
                if (tile + 2 == tiles) mask(next, tile + 1);
                float most = next[0][0];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < 2 * KB; ++u) {
                    if (u < 2 * KB - 1)
#pragma unroll
                        for (int db = 0; db < 4; ++db) vv[(u + 1) & 1][db] = Wave::value<4096>(Vt, v_at, u + 1, db);
                    const u32x4a pu = {pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]};
#pragma unroll
                    for (int db = 0; db < 4; ++db) w.o[db] = product(vv[u & 1][db], pu, w.o[db]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) most = fmaxf(most, next[u >> 1][(u & 1) * 8 + i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                top = halves_max(most) * a.scale_log2;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) s[kb] = next[kb];
            }
            store_both(tile + 1);
            ask_both(tile + 2);
            arrive(tile + 1);
        };
#pragma unroll 1
        for (int tile = 0; tile < tiles - 1; ++tile) step(tile);
        if (works) {
            w.raise(top);
            uint32_t pb[KB * 8];
#pragma unroll
            for (int i = 0; i < KB * 16; i += 2) pb[i / 2] = w.weigh<KB>(s, i, a.scale_log2);
            w.values<KB, 4096, true>(values_of(tiles - 1), v_at, pb);
        }
    }
    const float sum = halves_sum(w.sum);
    const int R = r.first + wave * 32 + col;
    if (R >= r.end) return;
    if (half == 0) a.part_ml[r.at + R] = (f32x2a){w.ref, sum};
    if (sum != 0.f) store_part(w, a.part_o + (r.at + R) * 128, half);
}

// A tail: its rows R, its token's positions, its keys.
struct Tail {
    int bi, head, R0, R1, length, p_low, p_high;
    int64_t sequence;
};
__device__ __forceinline__ Tail tail_of(const SharedArgs& a, int i) {
    Tail t;
    const AttendCall& c = a.c;
    const int tiles = a.by_kv.of(i), sequences = a.by_tail_tiles.of(tiles), tile = a.by_tail_tiles.rest(tiles, sequences), per = a.nt * c.group;
    t.head = a.by_kv.rest(i, tiles);
    t.bi = a.by_ns.of(sequences);
    const int s = a.by_ns.rest(sequences, t.bi);
    t.sequence = (int64_t)(a.b0 + t.bi) * a.share + a.s0 + s;
    t.length = __builtin_amdgcn_readfirstlane(c.lengths ? min(max(c.lengths[t.sequence], 0), c.n) : c.n);
    t.R0 = s * per + tile * kTile, t.R1 = s * per + min(per, (tile + 1) * kTile);
    t.p_low = t.length - c.m + a.t0 + a.by_group.of(tile * kTile);
    t.p_high = t.length - c.m + a.t0 + a.by_group.of(t.R1 - 1 - s * per);
    return t;
}
__device__ __forceinline__ Rows rows_of_tail(const SharedArgs& a, const Tail& t) { return {a.tail_at + ((int64_t)t.bi * a.c.kv + t.head) * a.rows, t.R0, t.R1}; }

// a / b of numbers below 2^53 (fewer steps than a division of 64 bits).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    const int64_t q = (int64_t)((double)a / (double)b);
    return q - (q * b > a) + ((q + 1) * b <= a);
}
// This workgroup's share of the kept rows: item(head of the slice, row tile, its number, kept rows, first and last tile of 64 keys).
template <class F>
__device__ __forceinline__ void each_item(const SharedArgs& a, int share, const F& item) {
    const int heads = a.nb * a.c.kv, lane = threadIdx.x & 63;
    const auto head_of = [&](int base) ALWAYS_INLINE { return base + lane < heads ? kept_rows(a, base + lane) : Kept{0, 0}; };
    Kept mine = head_of(0);
    int cost = cost_of(mine.count), sum = up_to(cost);
    int64_t total = __builtin_amdgcn_readlane(sum, 63), before = 0;
    for (int base = 64; base < heads; base += 64) total += __builtin_amdgcn_readlane(up_to(cost_of(head_of(base).count)), 63);
    total *= a.tiles;
    const int64_t per = quotient(total, a.shares), longer = total - per * a.shares;
    const int64_t low = per * share + min((int64_t)share, longer), high = per * (share + 1) + min((int64_t)share + 1, longer);
    if (low == high) return;
    for (int base = 0; base < heads && before * a.tiles < high; base += 64) {
        if (base > 0) mine = head_of(base), cost = cost_of(mine.count), sum = up_to(cost);
        const int64_t begin = (before + sum - cost) * a.tiles;     // of the head
        before += __builtin_amdgcn_readlane(sum, 63);
        for (uint64_t some = __ballot(cost > 0 && begin < high && begin + (int64_t)cost * a.tiles > low); some; some &= some - 1) {
            const int l = __builtin_ctzll(some), each = __builtin_amdgcn_readlane(cost, l), count = __builtin_amdgcn_readlane(mine.count, l);
            const int64_t from = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)begin, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(begin >> 32), l) << 32);
            const int64_t at = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)mine.at, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine.at >> 32), l) << 32);
            for (int tile = low > from ? (int)quotient(low - from, each) : 0; tile < a.tiles; ++tile) {
                const int64_t first = from + (int64_t)tile * each + kItemCost;      // where the tiles of keys begin
                if (first - kItemCost >= high) break;
                const int x = (int)min(max(low - first, (int64_t)0), (int64_t)(each - kItemCost)), y = (int)min(max(high - first, (int64_t)0), (int64_t)(each - kItemCost));
                if (x >= y) continue;
                if (threadIdx.x == 0 && x == 0) a.part_of_item[2 * ((base + l) * a.tiles + tile)] = share;
                if (threadIdx.x == 0 && y == each - kItemCost) a.part_of_item[2 * ((base + l) * a.tiles + tile) + 1] = share;
                item(base + l, tile, Kept{at, count}, x * 64, min(y * 64, count));
            }
        }
    }
}
// Where the partial results of share s and (head g, row tile) begin.
__device__ __forceinline__ int64_t part_of(const SharedArgs& a, int share, int g, int tile) { return ((int64_t)share + (int64_t)g * a.tiles + tile) * a.slot_rows; }

template <bool MX, int SETS>
__global__ __launch_bounds__(SETS * 64, 2) void attend_shared_kernel(SharedArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[SETS * 16384];
    __shared__ f32x2a ml[SETS][kTile];
    const AttendCall& c = a.c;
    const uint32_t lds_at = lds_address(&lds[0]);
    const int tid = threadIdx.x, col = tid & 31;
    int token;
    if (blockIdx.x < a.tail_blocks) {
        const int waves = a.tail_waves, of = __builtin_amdgcn_readfirstlane(tid >> 6) / waves;        // (the last tails may be none, and write nothing)
        const int64_t i = (int64_t)blockIdx.x * (SETS / waves) + of;
        const Tail t = tail_of(a, (int)min(i, a.tails - 1));
        Rows r = rows_of_tail(a, t);
        if (i >= a.tails) r.end = r.first;
        const char* row = (const char*)c.Q + query_row(a, t.bi, t.head, min(t.R0 + col, t.R1 - 1), &token) * 256;
        const int64_t from = (t.sequence * c.kv + t.head) * c.stride * 256;
        const char *K = (const char*)c.K + from, *V = (const char*)c.V + from;
        const int end = max(0, t.p_high + 1), p = t.length - c.m + token, at = of * waves * 16384;
        if (waves == 4) tail_rows<4>(a, tid & 255, lds + at, lds_at + at, ml + of * 4, K, V, end, p, t.p_low, row, r);
        else tail_rows<1>(a, tid & 63, lds + at, lds_at + at, nullptr, K, V, end, p, t.p_low, row, r);
        return;
    }
    // (neighbours in the list are neighbours in an XCD)
    const int block = (int)(blockIdx.x - a.tail_blocks), eighth = a.shares >> 3, share = block < eighth * 8 ? (block & 7) * eighth + (block >> 3) : block;
    each_item(a, share, [&](int g, int tile, const Kept& k, int begin, int end) ALWAYS_INLINE {
        const int bi = a.by_kv.of(g), head = a.by_kv.rest(g, bi), R = min(tile * (SETS * kTile) + (tid >> 6) * kTile + col, a.rows - 1);
        const char* row = (const char*)c.Q + query_row(a, bi, head, R, &token) * 256;
        const Rows r = {part_of(a, share, g, tile) - tile * (SETS * kTile), tile * (SETS * kTile), min(a.rows, (tile + 1) * (SETS * kTile))};
        const int width = MX ? 64 : 256;
        const char *K = (const char*)c.K_kept + k.at * width, *V = (const char*)c.V_kept + k.at * width;
        kept_rows_of<MX, SETS>(a, lds, lds_at, K, V, c.K_scales + k.at * 4, c.V_scales + k.at * 4, begin, end, row, r);
    });
}

// ---- fp32: a wave's 32 rows R, 32 keys at a time, operands straight from memory; the four waves take tiles in turn and are joined.  A wave has a unit to itself and 512 registers: a tile's
// values are on their way while its scores are made, and the next one's keys while the values are used.

// 32 keys' operands: of QK, at steps 0 .. 15, the channels of four number kStep step + kHalf half; of PV channel 32 db + lane % 32 of key i / 4 * 8 + i % 4 + 4 half.
template <bool MX> struct Operands32;
template <> struct Operands32<false> {
    static constexpr int kHalf = 1, kStep = 2;                     // fours of channels from half to half, and from step to step
    f32x4a k[16];
    float v[16][4];
    __device__ __forceinline__ void ask_keys(const char* K, const uint8_t*, int64_t row, int half) {
#pragma unroll
        for (int s = 0; s < 16; ++s) k[s] = ((const f32x4a*)(K + row * 512))[2 * s + half];
    }
    __device__ __forceinline__ void ask_values(const char* V, const uint8_t*, int64_t row, int i, int col) {
#pragma unroll
        for (int db = 0; db < 4; ++db) v[i][db] = ((const float*)(V + row * 512))[db * 32 + col];
    }
    // channels channel .. channel + 3 of a row of V
    static __device__ __forceinline__ f32x4a four(const char* V, const uint8_t*, int64_t row, int channel) { return *(const f32x4a*)((const float*)(V + row * 512) + channel); }
    __device__ __forceinline__ f32x4a key(int s) const { return k[s]; }
    __device__ __forceinline__ float value(int i, int db, int) const { return v[i][db]; }
};
template <> struct Operands32<true> {
    typedef uint32_t u32u __attribute__((aligned(1)));
    static constexpr int kHalf = 16, kStep = 1;
    u32x4a k[2];
    uint32_t k_scale[2], v_scale[16];
    uint8_t v[16][4];
    __device__ __forceinline__ void ask_keys(const char* K, const uint8_t* scales, int64_t row, int half) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            k[x] = ((const u32x4a*)(K + row * 64))[half * 2 + x];
            k_scale[x] = scales[row * 4 + half * 2 + x];
        }
    }
    __device__ __forceinline__ void ask_values(const char* V, const uint8_t* scales, int64_t row, int i, int col) {
        v_scale[i] = *(const u32u*)(scales + row * 4);
#pragma unroll
        for (int db = 0; db < 4; ++db) v[i][db] = ((const uint8_t*)V)[row * 64 + db * 16 + col / 2];
    }
    static __device__ __forceinline__ f32x4a four(const char* V, const uint8_t* scales, int64_t row, int channel) {
        const uint32_t codes = *(const uint16_t*)(V + row * 64 + channel / 2);
        const float unit = unit_of(scales[row * 4 + channel / 32]);
        const f32x2a x = two_f32<0>(codes, unit), y = two_f32<1>(codes, unit);
        return (f32x4a){x.x, x.y, y.x, y.y};
    }
    __device__ __forceinline__ f32x4a key(int s) const {
        const uint32_t codes = k[s >> 3][s >> 1 & 3];
        const float unit = unit_of(k_scale[s >> 3]);
        const f32x2a x = s & 1 ? two_f32<2>(codes, unit) : two_f32<0>(codes, unit), y = s & 1 ? two_f32<3>(codes, unit) : two_f32<1>(codes, unit);
        return (f32x4a){x.x, x.y, y.x, y.y};
    }
    __device__ __forceinline__ float value(int i, int db, int col) const {
        const f32x2a x = two_f32<0>(v[i][db], unit_of(v_scale[i] >> (8 * db) & 0xFF));
        return col & 1 ? x.y : x.x;
    }
};

template <bool MX, bool TAIL, int WAVES>
__device__ __forceinline__ void rows_f32(const SharedArgs& a, int tid, char* lds, f32x2a (*ml)[kTile], const char* K, const char* V, const uint8_t* K_scales, const uint8_t* V_scales, int begin, int end,
                                         int p, int p_low, const char* row, const Rows& r) {
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    typedef Operands32<MX> Operands;
    Operands from;
    f32x4a q[16];
    Wave w;                            // (its o, ref and sum)
    const int tiles = (end - begin + 31) / 32;
    const auto ask_keys = [&](int tile) ALWAYS_INLINE { from.ask_keys(K, K_scales, min(begin + tile * 32 + col, end - 1), half); };
    if (wave < tiles) ask_keys(wave);
    w.begin(row, half);
#pragma unroll
    for (int s = 0; s < 16; ++s) q[s] = ((const f32x4a*)row)[Operands::kStep * s + Operands::kHalf * half];
#pragma unroll 1
    for (int tile = wave; tile < tiles; tile += WAVES) {
        const int j0 = begin + tile * 32, count = min(32, end - j0);
#pragma unroll
        for (int i = 0; i < 16; ++i) from.ask_values(V, V_scales, j0 + min(i / 4 * 8 + i % 4 + half * 4, count - 1), i, col);
        __builtin_amdgcn_sched_barrier(0);
        f32x16a x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
        for (int s = 0; s < 16; ++s) {
            const f32x4a k = from.key(s);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[s][e], x, 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (tile + WAVES < tiles) ask_keys(tile + WAVES);
        const bool hidden = count < 32 || (TAIL && j0 + 31 > p_low);
        const int last = TAIL ? min(p, end - 1) : end - 1;
        if (hidden)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = j0 + i / 4 * 8 + i % 4 + half * 4 <= last ? x[i] : -INFINITY;
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
        top = halves_max(top) * a.scale_log2;
        if (__any(top > w.ref)) {
            const float next = top > w.ref ? top : w.ref, keep = next == w.ref ? 1.f : __builtin_amdgcn_exp2f(w.ref - next);
            w.sum *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db) w.o[db] *= keep;
            w.ref = next;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, -w.ref));
            w.sum += x[i];
        }
        const auto odd = [](float y) ALWAYS_INLINE { return (__float_as_uint(y) & 0x7F800000u) == 0x7F800000u; };
        if (!hidden) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int db = 0; db < 4; ++db) w.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(from.value(i, db, col), x[i], w.o[db], 0, 0, 0);
            continue;
        }
        // An infinity or NaN goes to the rows that see its key, whatever the weight, and meets no other's.
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const float y = from.value(i, db, col), z = i / 4 * 8 + i % 4 + half * 4 < count ? y : 0.f;
                bad |= odd(z);
                w.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(odd(z) ? 0.f : z, x[i], w.o[db], 0, 0, 0);
            }
        if (__any(bad))
#pragma unroll 1
            for (int key = 0; key < count; ++key)
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int n = 0; n < 16; n += 4) {
                        const f32x4a y = Operands::four(V, V_scales, j0 + key, db * 32 + n * 2 + half * 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j0 + key <= last && odd(y[e])) w.o[db][n + e] += y[e];
                    }
    }
    if constexpr (WAVES == 4) join_waves(w, tid, lds, ml, a.part_o, a.part_ml, r);
    else store_wave(a, w, r, col, half);
}

template <bool MX>
__global__ __launch_bounds__(256) void attend_shared_f32_kernel(SharedArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[65536];
    __shared__ f32x2a ml[4][kTile];
    const AttendCall& c = a.c;
    const int col = threadIdx.x & 31;
    int token;
    if (blockIdx.x < a.tail_blocks) {
        const int waves = a.tail_waves, of = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / waves;
        const int64_t i = (int64_t)blockIdx.x * (4 / waves) + of;
        const Tail t = tail_of(a, (int)min(i, a.tails - 1));
        Rows r = rows_of_tail(a, t);
        if (i >= a.tails) r.end = r.first;
        const char* row = (const char*)c.Q + query_row(a, t.bi, t.head, min(t.R0 + col, t.R1 - 1), &token) * 512;
        const int64_t at = (t.sequence * c.kv + t.head) * c.stride * 512;
        const char *K = (const char*)c.K + at, *V = (const char*)c.V + at;
        const int end = max(0, t.p_high + 1), p = t.length - c.m + token;
        if (waves == 4) rows_f32<false, true, 4>(a, threadIdx.x, lds, ml, K, V, nullptr, nullptr, 0, end, p, t.p_low, row, r);
        else rows_f32<false, true, 1>(a, threadIdx.x & 63, lds, ml, K, V, nullptr, nullptr, 0, end, p, t.p_low, row, r);
        return;
    }
    const int block = (int)(blockIdx.x - a.tail_blocks), eighth = a.shares >> 3, share = block < eighth * 8 ? (block & 7) * eighth + (block >> 3) : block;
    each_item(a, share, [&](int g, int tile, const Kept& k, int begin, int end) ALWAYS_INLINE {
        const char* row = (const char*)c.Q + query_row(a, a.by_kv.of(g), a.by_kv.rest(g, a.by_kv.of(g)), min(tile * kTile + col, a.rows - 1), &token) * 512;
        const int width = MX ? 64 : 512;
        rows_f32<MX, false, 4>(a, threadIdx.x, lds, ml, (const char*)c.K_kept + k.at * width, (const char*)c.V_kept + k.at * width, c.K_scales + k.at * 4, c.V_scales + k.at * 4, begin, end, 0, 0, row,
                            {part_of(a, share, g, tile) - tile * kTile, tile * kTile, min(a.rows, (tile + 1) * kTile)});
    });
}

// Joins the parts of four rows, a wave a row, two channels a lane: the shares that have tiles of its item, in order, and its tail's.
template <bool BF16>
__global__ __launch_bounds__(256) void attend_shared_join_kernel(SharedArgs a) {
    const AttendCall& c = a.c;
    const int g = a.by_quads.of(blockIdx.x), R = __builtin_amdgcn_readfirstlane(a.by_quads.rest(blockIdx.x, g) * 4 + (threadIdx.x >> 6));
    if (R >= a.rows) return;
    const int lane = threadIdx.x & 63, bi = a.by_kv.of(g), head = a.by_kv.rest(g, bi), tile = R / a.tile_rows, item = g * a.tiles + tile;
    const int first = a.part_of_item[2 * item], final = a.part_of_item[2 * item + 1];
    const bool any = kept_rows(a, g).count > 0;
    const int64_t at = part_of(a, 0, g, tile) + R - tile * a.tile_rows, tail = a.tail_at + (int64_t)g * a.rows + R;
    const f32x2a last = a.part_ml[tail], of_last = *(const f32x2a*)(a.part_o + tail * 128 + lane * 2);
    const int from = __builtin_amdgcn_readfirstlane(any ? first : 0), to = __builtin_amdgcn_readfirstlane(any ? final : -1);
    // 64 shares at a time, a lane each, then their rows of 512 bytes, sixteen on their way
    float ref = last.y == 0.f ? kNoScore : last.x;
    const auto rows_of = [&](f32x2a (&x)[16], int base, int many) ALWAYS_INLINE {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = *(const f32x2a*)(a.part_o + (at + (int64_t)(base + min(e, many - 1)) * a.slot_rows) * 128 + lane * 2);
    };
    f32x2a x[16];
    if (any) rows_of(x, from, min(16, to - from + 1));
    f32x2a ml = {0, 0};
    if (from + lane <= to) ml = a.part_ml[at + (int64_t)(from + lane) * a.slot_rows];
    if (ml.y != 0.f) ref = fmaxf(ref, ml.x);
    for (int s = from + 64 + lane; s <= to; s += 64) ref = fmaxf(ref, a.part_ml[at + (int64_t)s * a.slot_rows].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
    float sum = 0.f;
    f32x2a o = {0, 0};
    for (int base = from; base <= to; base += 64) {
        const int s = base + lane;
        if (base > from) {
            ml = (f32x2a){0, 0};
            if (s <= to) ml = a.part_ml[at + (int64_t)s * a.slot_rows];
        }
        const float weight = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - ref);
        sum += weight * ml.y;
        const uint64_t some = __ballot(ml.y != 0.f);               // (nothing seen: the row is not written)
        const int many = min(64, to - base + 1);
        for (int k = 0; k < many; k += 16) {
            if (base > from || k > 0) rows_of(x, base + k, min(16, many - k));
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (k + e < many && (some >> (k + e) & 1)) {
                    const float w = __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(weight), k + e));
                    o.x += w * x[e].x;
                    o.y += w * x[e].y;
                }
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (last.y != 0.f) {
        const float w = __builtin_amdgcn_exp2f(last.x - ref);
        sum += w * last.y;
        o.x += w * of_last.x;
        o.y += w * of_last.y;
    }
    const bool empty = sum == 0.f;
    const float over = empty ? 0.f : 1.f / sum;
    int token;
    const int64_t row = query_row(a, bi, head, R, &token);
    if (BF16) ((uint32_t*)c.out)[row * 64 + lane] = pack_bf16(o.x * over, o.y * over);
    else ((f32x2a*)c.out)[row * 64 + lane] = (f32x2a){o.x * over, o.y * over};
    if (c.lse && lane == 0) {
        const int s = a.by_per.of(R), in = a.by_per.rest(R, s);
        const int64_t sequence = (int64_t)(a.b0 + bi) * a.share + a.s0 + s;
        c.lse[(sequence * c.kv * c.group + head * c.group + a.by_group.rest(in, a.by_group.of(in))) * c.m + token] = empty ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

}  // namespace

hipError_t launch_attend_shared(const curdkv_ctx* ctx, const AttendCall& call, int share, hipStream_t stream) {
    SharedArgs a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.share = share;
    const bool bf16 = call.dtype == CURDKV_DTYPE_BF16, mx = call.K_scales != nullptr;
    // A slice's partial results, of its kept rows and its tails, have to lie in scratch: whole prefixes, else sequences of one, else tokens of one.  Rows R of a head fill tiles of
    // 128 or 256 (fp32: 32), and a share is a tile more.
    const int64_t room = (call.scratch_bytes - kScratchCounters) / (int64_t)(128 * sizeof(float) + sizeof(f32x2a));
    // Half of it is for the shares' parts, as far as one token's rows leave that much (11 prompts of 2393 rows, 27 answers of 5 tokens each: 707 us in one slice of 118 shares, 141 in three).
    const int64_t half = (room - 1024) / 2;
    const auto padded = [&](int64_t prefixes, int64_t sequences, int64_t tokens) {       // partial results of one share, and of the tails
        const int64_t rows = sequences * tokens * call.group, tile = !bf16 ? 32 : rows <= 128 ? 128 : 256;
        return prefixes * call.kv * ((rows <= tile ? rows : (rows + tile - 1) / tile * tile) + rows);
    };
    const auto fitting = [&](int64_t of, const auto& size) {       // the most of them that fit
        int64_t x = 1, y = of;                                     // x fits (cache_api.hip sees to one token of one sequence)
        while (x < y) {
            const int64_t z = (x + y + 1) / 2;
            if (size(z) <= half) x = z;
            else y = z - 1;
        }
        return x;
    };
    const int64_t tokens = fitting(call.m, [&](int64_t x) { return padded(1, 1, x); });
    const int64_t sequences = tokens < call.m ? 1 : fitting(share, [&](int64_t x) { return padded(1, x, tokens); });
    const int64_t prefixes = sequences < share ? 1 : fitting(call.count, [&](int64_t x) { return padded(x, sequences, tokens); });
    a.by_group = Divisor(call.group), a.by_kv = Divisor(call.kv);
    for (int64_t b = 0; b < call.count; b += prefixes)
        for (int64_t s = 0; s < share; s += sequences)
            for (int64_t t = 0; t < call.m; t += tokens) {
                a.b0 = (int)b, a.nb = (int)std::min(prefixes, call.count - b);
                a.s0 = (int)s, a.ns = (int)std::min<int64_t>(sequences, share - s);
                a.t0 = (int)t, a.nt = (int)std::min<int64_t>(tokens, call.m - t);
                a.rows = a.ns * a.nt * call.group;
                a.by_per = Divisor(a.nt * call.group);
                // Tiles of 256 rows, whose kept rows are read half as often, where there are twelve tiles of keys for every unit (64 answers: over 13107 rows 44 us so and 38 by 128, over 32768
                // 66 and 72, over 131072 177 and 197); of 128 also where there are fewer rows (16 answers over 13107: 28.3 us by 64, 26.7 so; 8 answers: 27.1 by 32, 22.5 so).
                const int64_t tiles_a_head = call.rows / (call.count * call.kv) / 64 + 1, heads = (int64_t)a.nb * call.kv;
                const int sets = !bf16 ? 1 : a.rows <= 128 || tiles_a_head * heads * ((a.rows + 255) / 256) < 12 * (int64_t)ctx->num_cu ? 4 : 8;
                a.tile_rows = sets * kTile;
                a.tiles = (a.rows + a.tile_rows - 1) / a.tile_rows;
                a.slot_rows = std::min(a.tile_rows, a.rows);
                a.tail_tiles = (a.nt * call.group + kTile - 1) / kTile;
                a.by_tail_tiles = Divisor(a.tail_tiles), a.by_ns = Divisor(a.ns), a.by_quads = Divisor((a.rows + 3) / 4);
                a.tails = (int64_t)a.nb * a.ns * call.kv * a.tail_tiles;
                // One wave a tail: where there is no more than a tile of it, or where tails keep all waves busy (7 prompts' 45 answers of up to 8 tokens 50 us by four waves, 31 by one; 16
                // prompts' 16 of up to 130 86 and 76; 8 prompts' 16 of 500, half as many, 81 and 88).
                a.tail_waves = call.n <= 32 || a.tails >= (call.n <= 256 ? 4 : 8) * (int64_t)ctx->num_cu ? 1 : 4;
                a.tail_blocks = (a.tails * a.tail_waves + std::max(sets, 4) - 1) / std::max(sets, 4);
                // Shares of the kept rows, by their cost: four tiles of 64 keys each (two, up to 64 shares), up to a workgroup a unit; eight, up to two a unit (256 rows, and fp32, whose registers
                // fill it: one), as far as there is scratch.  (16 answers over 13107 rows: 28.3 us with four tiles up to two workgroups, 24.0 so; over 300 rows 18.6 with four tiles, 13.8 so;
                // fp32, 13107 rows: 66 with two workgroups, 53 so.)
                const int64_t items = heads * a.tiles, tail_rows = heads * a.rows, tiles = (tiles_a_head + kItemCost) * items;
                const int64_t useful = std::max({std::min<int64_t>(64, tiles / 2), std::min<int64_t>(ctx->num_cu, tiles / 4), tiles / 8});
                const int64_t units = (sets == 4 ? 2 : 1) * (int64_t)ctx->num_cu;
                a.shares = (int)std::max<int64_t>(1, std::min({useful, units, (room - 1024 - tail_rows) / a.slot_rows - items}));
                a.tail_at = (a.shares + items) * a.slot_rows;
                a.part_o = (float*)((char*)call.scratch + kScratchCounters);
                a.part_ml = (f32x2a*)(a.part_o + (a.tail_at + tail_rows) * 128);
                a.part_of_item = (int32_t*)(a.part_ml + a.tail_at + tail_rows);
                const auto launch = [&](auto kernel) { kernel<<<(unsigned)(a.tail_blocks + a.shares), sets > 4 ? 512 : 256, 0, stream>>>(a); };
                if (!bf16) mx ? launch(attend_shared_f32_kernel<true>) : launch(attend_shared_f32_kernel<false>);
                else if (sets == 8) mx ? launch(attend_shared_kernel<true, 8>) : launch(attend_shared_kernel<false, 8>);
                else mx ? launch(attend_shared_kernel<true, 4>) : launch(attend_shared_kernel<false, 4>);
                const unsigned joins = (unsigned)((int64_t)a.nb * call.kv * ((a.rows + 3) / 4));
                if (bf16) attend_shared_join_kernel<true><<<joins, 256, 0, stream>>>(a);
                else attend_shared_join_kernel<false><<<joins, 256, 0, stream>>>(a);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
    return hipSuccess;
}

}  // namespace curdkv
