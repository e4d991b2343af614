// Attention of many sequences over the kept rows that they share, and over their own tails: of two sets of keys with (M1, L1, o1) and (M2, L2, o2), o un-normalised,
// the whole has M = max, L = L1 2^(M1-M) + L2 2^(M2-M) and o likewise (scores in units of log 2).  So the rows R of all of a prefix's
// sequences (R = (sequence, token, head)) stand side by side over its kept rows, which are read once for 128 of them (or 32), each
// sequence's own over its tail, and a second kernel joins what they found.
//
// One launch: workgroups of kept rows (a prefix's KV head, 128 or 32 rows R, a part of the keys), then those of tails (a sequence's KV head, 32 rows R).
// S^T = K Q^T and O^T = V^T P^T by mfma_f32_32x32x16_bf16, operands and layout of the tiles in LDS as in attend_prompt.hip: columns of 64 bytes a row, V read transposed, P from
// the registers that S^T leaves it in.  With 128 rows the four waves have 32 each and share tiles of 64 keys; with 32 each wave has tiles of 32 keys of its own and the waves are joined
// in LDS.  Rows in 4 bits are expanded on their way into LDS, exactly.
// fp32: mfma_f32_32x32x2, operands straight from memory.

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
    int rows, tiles;                   // of a prefix's KV head: ns * nt * group, and tiles of kTile (or 4 kTile) of them
    int parts;                         // that its kept rows are shared out over
    int tail_tiles;                    // of a sequence's nt * group rows
    int64_t kept_blocks, slots;        // slots: rows R of all heads, nb * kv * rows
    float* part_o;                     // [parts + 1][slots][128], un-normalised; part `parts` is the tail's
    f32x2a* part_ml;                   // the same of reference points and sums; sum 0: nothing seen, o not written
};

// Rows R of a workgroup: first + col of `rows` of prefix g's head, or of one sequence's.
struct Rows {
    int64_t slot;                      // of row 0
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
    const int per = a.nt * a.c.group, s = R / per, t = R % per / a.c.group;
    *token = a.t0 + t;
    return ((((int64_t)(a.b0 + bi) * a.share + a.s0 + s) * a.c.m + a.t0 + t) * a.c.kv + head) * a.c.group + R % a.c.group;
}

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
    template <int KB>
    __device__ __forceinline__ void scores(const char* Kt, int col, int half, f32x16a (&x)[KB]) const {
        const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kb][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[kb] = product(*(const u32x4a*)(Kt + k_at[i & 1] + (i >> 1) * (KB * 2048) + kb * 2048), q[i], x[kb]);
        }
    }
    // scores -> weights (relative to `ref`, which moves when it lies too far below), pairs of bf16 in the order of the next product
    template <int KB>
    __device__ __forceinline__ void weigh(f32x16a (&x)[KB], float scale_log2, uint32_t (&pb)[KB * 8]) {
        float top = x[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
        top = halves_max(top) * scale_log2;
        if (__any(top > ref + kLoose)) {
            const float next = top > ref + kLoose ? top : ref, keep = next == ref ? 1.f : __builtin_amdgcn_exp2f(ref - next);
            sum *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db) o[db] *= keep;
            ref = next;
        }
#pragma unroll
        for (int i = 0; i < KB * 16; i += 2) {
            const float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 4][i & 15], scale_log2, -ref));
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 4][(i & 15) + 1], scale_log2, -ref));
            sum += u + v;
            pb[i / 2] = pack_bf16(u, v);
        }
    }
    template <int KB, bool FINITE>     // !FINITE: zeros in the place of infinities and NaN
    __device__ __forceinline__ void values(const char* Vt, int v_at, const uint32_t (&pb)[KB * 8]) {
#pragma unroll
        for (int u = 0; u < KB * 2; ++u)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const char* p = Vt + v_at + db * (KB * 2048) + u * 1024;
                const u32x2 x = read_transposed(p), y = read_transposed(p + 512);
                u32x4a w = {x.x, x.y, y.x, y.y};
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

// Where tiles of 32 KB keys come from, into LDS as four columns of 64 bytes a row (K's pieces of 16 bytes permuted by (row / 2) % 4); keys `begin` .. `end` - 1 of rows
// at K, V.  PER: tiles between this wave's (each wave its own, LANES = 64) or 1 (all four waves together, LANES = 256).
__device__ __forceinline__ uint32_t piece_at(int row, int column, int piece, bool keys, int keys_of_tile) {
    return column * (keys_of_tile * 64) + row * 64 + ((keys ? piece ^ ((row >> 1) & 3) : piece) << 4);
}
// 1 KB blocks of 16 rows' columns, block first .. first + COUNT - 1 of a tile, straight into LDS.
template <int KEYS, int COUNT>
__device__ __forceinline__ void fetch_bf16(uint32_t lds, const char* rows, int count, bool keys, int first, int lane) {
    rows = (const char*)uniform((int64_t)rows);
    lds = __builtin_amdgcn_readfirstlane(lds);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int block = first + i, column = block / (KEYS / 16), row = block % (KEYS / 16) * 16 + (lane >> 2), piece = lane & 3;
        dma16(lds + block * 1024, rows, min(row, count - 1) * 256 + column * 64 + ((keys ? piece ^ ((row >> 1) & 3) : piece) << 4));
    }
}
// Rows in 4 bits: a lane's share of a tile, 16 or 32 bytes of codes of one row, and its scales.
template <int BLOCKS>
struct Codes {
    u32x4a codes[BLOCKS];
    uint32_t scales[BLOCKS];
    __device__ __forceinline__ void load(const uint8_t* rows, const uint8_t* scale, int64_t row, int column) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            codes[i] = *(const u32x4a*)(rows + row * 64 + (column + i) * 16);
            scales[i] = scale[row * 4 + column + i];
        }
    }
    __device__ __forceinline__ void store(char* tile, int row, int column, bool keys, int keys_of_tile) const {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int p = 0; p < 4; ++p) *(u32x4a*)(tile + piece_at(row, column + i, p, keys, keys_of_tile)) = eight_bf16(codes[i][p], unit_of(scales[i]));
    }
};

// Zeros in rows count .. KEYS - 1 of a tile of V, by LANES threads.
template <int KEYS, int LANES>
__device__ __forceinline__ void clear_beyond(char* tile, int count, int thread) {
    for (int i = count * 16 + thread; i < KEYS * 16; i += LANES) *(u32x4a*)(tile + (i & 3) * (KEYS * 64) + (i >> 4) * 64 + (i >> 2 & 3) * 16) = (u32x4a){0, 0, 0, 0};
}

// A partial result of 32 rows R: O^T's lanes (column R, channels 32 db + 8 i + 4 half ..) to rows of 128 floats.
__device__ __forceinline__ void store_part(const Wave& w, float* to, int half, float scale) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4a*)(to + db * 32 + i * 8 + half * 4) = (f32x4a){w.o[db][4 * i] * scale, w.o[db][4 * i + 1] * scale, w.o[db][4 * i + 2] * scale, w.o[db][4 * i + 3] * scale};
}

// The parts of four waves over the same 32 rows R, through 64 KB of LDS: one partial result.
__device__ __forceinline__ void join_waves(Wave& w, char* lds, f32x2a (*ml)[kTile], float* part_o, f32x2a* part_ml, const Rows& r) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const float sum = halves_sum(w.sum);
    if (half == 0) ml[wave][col] = (f32x2a){w.ref, sum};
    __syncthreads();                   // (and nobody reads tiles any more)
    float ref = ml[0][col].x;
#pragma unroll
    for (int k = 1; k < 4; ++k) ref = fmaxf(ref, ml[k][col].x);
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
    float m = ml[0][row].x, l = 0.f;
#pragma unroll
    for (int k = 1; k < 4; ++k) m = fmaxf(m, ml[k][row].x);
#pragma unroll
    for (int k = 0; k < 4; ++k) l += ml[k][row].y == 0.f ? 0.f : ml[k][row].y * __builtin_amdgcn_exp2f(ml[k][row].x - m);
    if ((tid & 7) == 0) part_ml[r.slot + R] = (f32x2a){m, l};
    if (l == 0.f) return;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int piece = (tid & 7) + p * 8;
        f32x4a x = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) x += *(const f32x4a*)((const float*)lds + (k * kTile + row) * 128 + (piece ^ (row & 7)) * 4);
        *(f32x4a*)(part_o + (r.slot + R) * 128 + piece * 4) = x;
    }
}

// Tokens' positions hide a tail's later rows: key j is seen at p where j <= p.
// A tile that some row of the 32 does not see whole, by one wave: infinities and NaN among its values must not meet the zero weights of rows that do not see them.
template <int KB>
__device__ __forceinline__ void hidden_step(Wave& w, const char* Kt, const char* Vt, int v_at, int j0, int p, float scale_log2, int col, int half, int lane) {
    f32x16a s[KB];
    w.scores<KB>(Kt, col, half, s);
    const int far = p - j0 - half * 4;
#pragma unroll
    for (int i = 0; i < KB * 16; ++i) s[i >> 4][i & 15] = (i >> 4) * 32 + (i & 15) / 4 * 8 + i % 4 <= far ? s[i >> 4][i & 15] : -INFINITY;
    uint32_t pb[KB * 8];
    w.weigh<KB>(s, scale_log2, pb);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < KB * 8; ++i) {
        const u32x4a x = *(const u32x4a*)(Vt + i * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7F80u) == 0x7F80u || (x[e] & 0x7F800000u) == 0x7F800000u;
    }
    if (!__any(bad)) {
        w.values<KB, true>(Vt, v_at, pb);
        return;
    }
    w.values<KB, false>(Vt, v_at, pb);
    for (int key = 0; key < KB * 32; ++key) {
        if (key > p - j0) break;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x2 v = *(const u32x2*)(Vt + db * (KB * 2048) + key * 64 + i * 16 + half * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t x = e % 2 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16;
                    if ((x & 0x7F800000u) == 0x7F800000u) w.o[db][4 * i + e] += __uint_as_float(x);
                }
            }
    }
}

// 32 rows R, each wave over tiles of 32 keys of its own.  TAIL: row R's token stands at p.
template <bool MX, bool TAIL>
__device__ __forceinline__ void few_rows(const SharedArgs& a, char* lds, f32x2a (*ml)[kTile], const void* K, const void* V, const uint8_t* K_scales, const uint8_t* V_scales,
                                         int begin, int end, int p, int p_low, const char* row, const Rows& r, float* part_o, f32x2a* part_ml) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int v_at = (4 * half + l16 / 4) * 64 + (lane >> 4 & 1) * 32 + (l16 & 3) * 8;
    char *Kt = lds + wave * 16384, *Vt = Kt + 8192;
    const uint32_t k_lds = lds_address(Kt), v_lds = lds_address(Vt);
    Wave w;
    w.begin(row, half);
    const int tiles = (end - begin + 31) / 32;
    for (int tile = wave; tile < tiles; tile += 4) {
        const int j0 = begin + tile * 32, count = min(32, end - j0);
        if constexpr (MX) {
            Codes<2> k, v;
            const int at = min(lane >> 1, count - 1);
            k.load((const uint8_t*)K, K_scales, j0 + at, (lane & 1) * 2);
            v.load((const uint8_t*)V, V_scales, j0 + at, (lane & 1) * 2);
            k.store(Kt, lane >> 1, (lane & 1) * 2, true, 32);
            v.store(Vt, lane >> 1, (lane & 1) * 2, false, 32);
        } else {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch_bf16<32, 8>(k_lds, (const char*)K + (int64_t)j0 * 256, count, true, 0, lane);
            fetch_bf16<32, 8>(v_lds, (const char*)V + (int64_t)j0 * 256, count, false, 0, lane);
            dma_wait();
        }
        if (count < 32) clear_beyond<32, 64>(Vt, count, lane);
        if (count < 32 || (TAIL && j0 + 31 > p_low)) {
            hidden_step<1>(w, Kt, Vt, v_at, j0, TAIL ? min(p, end - 1) : end - 1, a.scale_log2, col, half, lane);
            continue;
        }
        f32x16a s[1];
        uint32_t pb[8];
        w.scores<1>(Kt, col, half, s);
        w.weigh<1>(s, a.scale_log2, pb);
        w.values<1, true>(Vt, v_at, pb);
    }
    __syncthreads();
    join_waves(w, lds, ml, part_o, part_ml, r);
}

// 128 rows R, 32 a wave, tiles of 64 keys for all.
template <bool MX>
__device__ __forceinline__ void many_rows(const SharedArgs& a, char* lds, const void* K, const void* V, const uint8_t* K_scales, const uint8_t* V_scales, int begin, int end,
                                          const char* row, const Rows& r, float* part_o, f32x2a* part_ml) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int v_at = (4 * half + l16 / 4) * 64 + (lane >> 4 & 1) * 32 + (l16 & 3) * 8;
    Wave w;
    w.begin(row, half);
    const int tiles = (end - begin + 63) / 64;
    const auto count_of = [&](int tile) ALWAYS_INLINE { return min(64, end - begin - tile * 64); };
    Codes<1> k, v;
    const auto ask = [&](int tile) ALWAYS_INLINE {         // 4 bits: this thread's share into registers; bf16: the wave's on its way into LDS
        const int64_t j0 = begin + tile * 64;
        if constexpr (MX) {
            const int at = min(tid >> 2, count_of(tile) - 1);
            k.load((const uint8_t*)K, K_scales, j0 + at, tid & 3);
            v.load((const uint8_t*)V, V_scales, j0 + at, tid & 3);
        } else {
            char* to = lds + (tile & 1) * 32768;
            fetch_bf16<64, 4>(lds_address(to), (const char*)K + j0 * 256, count_of(tile), true, wave * 4, lane);
            fetch_bf16<64, 4>(lds_address(to + 16384), (const char*)V + j0 * 256, count_of(tile), false, wave * 4, lane);
        }
    };
    const auto arrive = [&](int tile) ALWAYS_INLINE {
        char* to = lds + (tile & 1) * 32768;
        if constexpr (MX) {
            k.store(to, tid >> 2, tid & 3, true, 64);
            v.store(to + 16384, tid >> 2, tid & 3, false, 64);
        } else {
            dma_wait();
        }
        if (count_of(tile) < 64) {
            __syncthreads();
            clear_beyond<64, 256>(to + 16384, count_of(tile), tid);
        }
        __syncthreads();
    };
    if (tiles > 0) {
        ask(0);
        arrive(0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) loaded(w.q[i]);
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) ask(tile + 1);
        const char *Kt = lds + (tile & 1) * 32768, *Vt = Kt + 16384;
        f32x16a s[2];
        uint32_t pb[16];
        w.scores<2>(Kt, col, half, s);
        const int count = count_of(tile);
        if (count < 64) {
            const int far = count - 1 - half * 4;
#pragma unroll
            for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = (i >> 4) * 32 + (i & 15) / 4 * 8 + i % 4 <= far ? s[i >> 4][i & 15] : -INFINITY;
        }
        w.weigh<2>(s, a.scale_log2, pb);
        w.values<2, true>(Vt, v_at, pb);
        if (tile + 1 < tiles) arrive(tile + 1);
    }
    const float sum = halves_sum(w.sum);
    const int R = r.first + wave * 32 + col;
    if (R >= r.end) return;
    if (half == 0) part_ml[r.slot + R] = (f32x2a){w.ref, sum};
    if (sum != 0.f) store_part(w, part_o + (r.slot + R) * 128, half, 1.f);
}

// The kept rows of prefix head g of the slice that part `part` has: [begin, end) of the arrays.
struct Kept {
    int64_t at;                        // of row 0
    int begin, end;
};
__device__ __forceinline__ Kept kept_rows(const SharedArgs& a, int g, int part) {
    const AttendCall& c = a.c;
    const int64_t* offsets = c.offsets + (int64_t)a.b0 * c.kv + g;
    const int64_t begin = min(max(offsets[0], (int64_t)0), c.total), count = min(max(offsets[1], begin), c.total) - begin, tiles = (count + 63) / 64;
    return {uniform(begin), __builtin_amdgcn_readfirstlane((int)(tiles * part / a.parts * 64)),
            __builtin_amdgcn_readfirstlane((int)min(count, tiles * (part + 1) / a.parts * 64))};
}

template <bool MX, bool MANY>
__global__ __launch_bounds__(256, 2) void attend_shared_kernel(SharedArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[65536];
    __shared__ f32x2a ml[4][kTile];
    const AttendCall& c = a.c;
    const int tid = threadIdx.x, col = tid & 31;
    if (blockIdx.x < a.kept_blocks) {
        constexpr int kRows = MANY ? 4 * kTile : kTile;
        const int heads = a.nb * c.kv, g = blockIdx.x % heads, part = blockIdx.x / heads % a.parts, tile = blockIdx.x / heads / a.parts;
        const int bi = g / c.kv, head = g % c.kv, R = min(tile * kRows + (MANY ? (tid >> 6) * 32 : 0) + col, a.rows - 1);
        int token;
        const char* row = (const char*)c.Q + query_row(a, bi, head, R, &token) * 256;
        const Rows r = {(int64_t)g * a.rows, tile * kRows, a.rows};
        const Kept k = kept_rows(a, g, part);
        const int width = MX ? 64 : 256;
        const char *K = (const char*)c.K_kept + k.at * width, *V = (const char*)c.V_kept + k.at * width;
        float* part_o = a.part_o + part * a.slots * 128;
        f32x2a* part_ml = a.part_ml + part * a.slots;
        if constexpr (MANY) many_rows<MX>(a, lds, K, V, c.K_scales + k.at * 4, c.V_scales + k.at * 4, k.begin, k.end, row, r, part_o, part_ml);
        else few_rows<MX, false>(a, lds, ml, K, V, c.K_scales + k.at * 4, c.V_scales + k.at * 4, k.begin, k.end, 0, 0, row, r, part_o, part_ml);
        return;
    }
    const int64_t i = blockIdx.x - a.kept_blocks;
    const int head = (int)(i % c.kv), tile = (int)(i / c.kv % a.tail_tiles), s = (int)(i / c.kv / a.tail_tiles % a.ns), bi = (int)(i / c.kv / a.tail_tiles / a.ns);
    const int64_t sequence = (int64_t)(a.b0 + bi) * a.share + a.s0 + s;
    const int per = a.nt * c.group, length = __builtin_amdgcn_readfirstlane(c.lengths ? min(max(c.lengths[sequence], 0), c.n) : c.n);
    const int R0 = s * per + tile * kTile, R1 = s * per + min(per, (tile + 1) * kTile);
    int token;
    const char* row = (const char*)c.Q + query_row(a, bi, head, min(R0 + col, R1 - 1), &token) * 256;
    const int p = length - c.m + token, p_low = length - c.m + a.t0 + tile * kTile / c.group, p_high = length - c.m + a.t0 + (R1 - 1 - s * per) / c.group;
    const Rows r = {((int64_t)bi * c.kv + head) * a.rows, R0, R1};
    const int64_t from = (sequence * c.kv + head) * c.stride * 256;
    few_rows<false, true>(a, lds, ml, (const char*)c.K + from, (const char*)c.V + from, nullptr, nullptr, 0, max(0, p_high + 1), p, p_low, row, r,
                          a.part_o + a.parts * a.slots * 128, a.part_ml + a.parts * a.slots);
}

// ---- fp32: a wave's 32 rows R, 32 keys at a time, operands straight from memory; the four waves take tiles in turn and are joined.
template <bool MX>
struct Source32 {                      // keys' rows of one head
    const char *K, *V;
    const uint8_t *K_scales, *V_scales;
    // channels of row j that QK's operand has in this half: 4 at step s (0 .. 15)
    __device__ __forceinline__ f32x4a key(int j, int s, int half) const {
        if constexpr (MX) {
            const uint32_t codes = ((const uint16_t*)K)[(int64_t)j * 32 + 2 * s + half];
            const float unit = unit_of(K_scales[(int64_t)j * 4 + s / 4]);
            const f32x2a x = two_f32<0>(codes, unit), y = two_f32<1>(codes, unit);
            return (f32x4a){x.x, x.y, y.x, y.y};
        } else {
            return ((const f32x4a*)(K + (int64_t)j * 512))[2 * s + half];
        }
    }
    __device__ __forceinline__ float value(int j, int channel) const {
        if constexpr (MX) {
            const uint32_t codes = ((const uint8_t*)V)[(int64_t)j * 64 + channel / 2];
            const f32x2a x = two_f32<0>(codes, unit_of(V_scales[(int64_t)j * 4 + channel / 32]));
            return channel & 1 ? x.y : x.x;
        } else {
            return ((const float*)(V + (int64_t)j * 512))[channel];
        }
    }
};

template <bool MX, bool TAIL>
__device__ __forceinline__ void rows_f32(const SharedArgs& a, char* lds, f32x2a (*ml)[kTile], const Source32<MX>& from, int begin, int end, int p, int p_low,
                                         const char* row, const Rows& r, float* part_o, f32x2a* part_ml) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    f32x4a q[16];
    Wave w;                            // (its o, ref and sum)
    w.begin(row, half);
#pragma unroll
    for (int s = 0; s < 16; ++s) q[s] = ((const f32x4a*)row)[2 * s + half];
    const int tiles = (end - begin + 31) / 32;
    for (int tile = wave; tile < tiles; tile += 4) {
        const int j0 = begin + tile * 32, count = min(32, end - j0);
        f32x16a x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
        for (int s = 0; s < 16; ++s) {
            const f32x4a k = from.key(j0 + min(col, count - 1), s, half);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[s][e], x, 0, 0, 0);
        }
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
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int key = i / 4 * 8 + i % 4 + half * 4;  // of this half
            float v[4];
            bool bad = false;
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                v[db] = key < count ? from.value(j0 + min(key, count - 1), db * 32 + col) : 0.f;
                bad |= (__float_as_uint(v[db]) & 0x7F800000u) == 0x7F800000u;
            }
            if (hidden && __any(bad)) {
                // Such a value goes to the rows that see its key, whatever the weight: column R is lane % 32, and the value of channel 32 db + n is lane n's of the key's half.
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    const bool sees_it = j0 + i / 4 * 8 + i % 4 + h * 4 <= last;
#pragma unroll
                    for (int db = 0; db < 4; ++db)
#pragma unroll
                        for (int n = 0; n < 16; ++n) {
                            const float y = __shfl(v[db], h * 32 + n / 4 * 8 + n % 4 + half * 4);
                            if ((__float_as_uint(y) & 0x7F800000u) == 0x7F800000u && sees_it) w.o[db][n] += y;
                        }
                }
#pragma unroll
                for (int db = 0; db < 4; ++db)
                    if ((__float_as_uint(v[db]) & 0x7F800000u) == 0x7F800000u) v[db] = 0.f;
            }
#pragma unroll
            for (int db = 0; db < 4; ++db) w.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[db], x[i], w.o[db], 0, 0, 0);
        }
    }
    __syncthreads();
    join_waves(w, lds, ml, part_o, part_ml, r);
}

template <bool MX>
__global__ __launch_bounds__(256) void attend_shared_f32_kernel(SharedArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[65536];
    __shared__ f32x2a ml[4][kTile];
    const AttendCall& c = a.c;
    const int col = threadIdx.x & 31;
    int token;
    if (blockIdx.x < a.kept_blocks) {
        const int heads = a.nb * c.kv, g = blockIdx.x % heads, part = blockIdx.x / heads % a.parts, tile = blockIdx.x / heads / a.parts;
        const char* row = (const char*)c.Q + query_row(a, g / c.kv, g % c.kv, min(tile * kTile + col, a.rows - 1), &token) * 512;
        const Kept k = kept_rows(a, g, part);
        const int width = MX ? 64 : 512;
        const Source32<MX> from = {(const char*)c.K_kept + k.at * width, (const char*)c.V_kept + k.at * width, c.K_scales + k.at * 4, c.V_scales + k.at * 4};
        rows_f32<MX, false>(a, lds, ml, from, k.begin, k.end, 0, 0, row, {(int64_t)g * a.rows, tile * kTile, a.rows}, a.part_o + part * a.slots * 128,
                            a.part_ml + part * a.slots);
        return;
    }
    const int64_t i = blockIdx.x - a.kept_blocks;
    const int head = (int)(i % c.kv), tile = (int)(i / c.kv % a.tail_tiles), s = (int)(i / c.kv / a.tail_tiles % a.ns), bi = (int)(i / c.kv / a.tail_tiles / a.ns);
    const int64_t sequence = (int64_t)(a.b0 + bi) * a.share + a.s0 + s;
    const int per = a.nt * c.group, length = __builtin_amdgcn_readfirstlane(c.lengths ? min(max(c.lengths[sequence], 0), c.n) : c.n);
    const int R0 = s * per + tile * kTile, R1 = s * per + min(per, (tile + 1) * kTile);
    const char* row = (const char*)c.Q + query_row(a, bi, head, min(R0 + col, R1 - 1), &token) * 512;
    const int p = length - c.m + token, p_low = length - c.m + a.t0 + tile * kTile / c.group, p_high = length - c.m + a.t0 + (R1 - 1 - s * per) / c.group;
    const int64_t at = (sequence * c.kv + head) * c.stride * 512;
    rows_f32<false, true>(a, lds, ml, Source32<false>{(const char*)c.K + at, (const char*)c.V + at, nullptr, nullptr}, 0, max(0, p_high + 1), p, p_low, row,
                          {((int64_t)bi * c.kv + head) * a.rows, R0, R1}, a.part_o + a.parts * a.slots * 128, a.part_ml + a.parts * a.slots);
}

// Joins the parts of four rows, a wave a row, two channels a lane.
template <bool BF16>
__global__ __launch_bounds__(256) void attend_shared_join_kernel(SharedArgs a) {
    const AttendCall& c = a.c;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= a.slots) return;
    const int lane = threadIdx.x & 63, g = (int)(at / a.rows), R = (int)(at - (int64_t)g * a.rows), head = g % c.kv;
    float ref = kNoScore, sum = 0.f;
    for (int k = 0; k <= a.parts; ++k) ref = fmaxf(ref, a.part_ml[at + k * a.slots].x);
    f32x2a o = {0, 0};
    for (int k = 0; k <= a.parts; ++k) {
        const f32x2a ml = a.part_ml[at + k * a.slots];
        if (ml.y == 0.f) continue;     // (nothing seen, o not written)
        const f32x2a x = *(const f32x2a*)(a.part_o + (at + k * a.slots) * 128 + lane * 2);
        const float weight = __builtin_amdgcn_exp2f(ml.x - ref);
        sum += weight * ml.y;
        o.x += weight * x.x;
        o.y += weight * x.y;
    }
    const bool empty = sum == 0.f;
    const float over = empty ? 0.f : 1.f / sum;
    int token;
    const int64_t row = query_row(a, g / c.kv, head, R, &token);
    if (BF16) ((uint32_t*)c.out)[row * 64 + lane] = pack_bf16(o.x * over, o.y * over);
    else ((f32x2a*)c.out)[row * 64 + lane] = (f32x2a){o.x * over, o.y * over};
    if (c.lse && lane == 0) {
        const int64_t sequence = (int64_t)(a.b0 + g / c.kv) * a.share + a.s0 + R / (a.nt * c.group);
        c.lse[(sequence * c.kv * c.group + head * c.group + R % c.group) * c.m + token] = empty ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

}  // namespace

hipError_t launch_attend_shared(const curdkv_ctx* ctx, const AttendCall& call, int share, hipStream_t stream) {
    SharedArgs a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.share = share;
    const bool bf16 = call.dtype == CURDKV_DTYPE_BF16, mx = call.K_scales != nullptr;
    // A slice's partial results, of its kept rows and its tails, have to lie in scratch: whole prefixes, else sequences of one, else tokens of one.
    const int64_t room = (call.scratch_bytes - kScratchCounters) / (int64_t)(128 * sizeof(float) + sizeof(f32x2a)) / 2;
    const int64_t heads = (int64_t)call.kv * call.group;
    const int64_t tokens = std::min<int64_t>(call.m, room / heads), sequences = tokens < call.m ? 1 : std::min<int64_t>(share, room / (heads * tokens));
    const int64_t prefixes = sequences < share ? 1 : std::min<int64_t>(call.count, room / (heads * tokens * sequences));
    for (int64_t b = 0; b < call.count; b += prefixes)
        for (int64_t s = 0; s < share; s += sequences)
            for (int64_t t = 0; t < call.m; t += tokens) {
                a.b0 = (int)b, a.nb = (int)std::min(prefixes, call.count - b);
                a.s0 = (int)s, a.ns = (int)std::min<int64_t>(sequences, share - s);
                a.t0 = (int)t, a.nt = (int)std::min<int64_t>(tokens, call.m - t);
                a.rows = a.ns * a.nt * call.group;
                const bool many = bf16 && a.rows > kTile;
                a.tiles = (a.rows + (many ? 4 : 1) * kTile - 1) / ((many ? 4 : 1) * kTile);
                a.tail_tiles = (a.nt * call.group + kTile - 1) / kTile;
                a.slots = (int64_t)a.nb * call.kv * a.rows;
                // Parts of the kept rows until every unit has two workgroups, 4 tiles of 64 keys each at least, as far as there is scratch.
                const int64_t blocks = (int64_t)a.nb * call.kv * a.tiles, tiles = call.rows / (call.count * call.kv) / 64;
                a.parts = (int)std::max<int64_t>(1, std::min(std::min(2 * ctx->num_cu / blocks, tiles / 4), 2 * room / a.slots - 1));
                a.kept_blocks = blocks * a.parts;
                a.part_o = (float*)((char*)call.scratch + kScratchCounters);
                a.part_ml = (f32x2a*)(a.part_o + (a.parts + 1) * a.slots * 128);
                const int64_t all = a.kept_blocks + (int64_t)a.nb * a.ns * call.kv * a.tail_tiles;
                const auto launch = [&](auto kernel) { kernel<<<(unsigned)all, 256, 0, stream>>>(a); };
                if (!bf16) mx ? launch(attend_shared_f32_kernel<true>) : launch(attend_shared_f32_kernel<false>);
                else if (many) mx ? launch(attend_shared_kernel<true, true>) : launch(attend_shared_kernel<false, true>);
                else mx ? launch(attend_shared_kernel<true, false>) : launch(attend_shared_kernel<false, false>);
                const unsigned joins = (unsigned)((a.slots + 3) / 4);
                if (bf16) attend_shared_join_kernel<true><<<joins, 256, 0, stream>>>(a);
                else attend_shared_join_kernel<false><<<joins, 256, 0, stream>>>(a);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
    return hipSuccess;
}

}  // namespace curdkv
