// Attention of many tokens over an fp32 cache: as attend_prompt.hip, with every factor in three parts of 8 bits, x = h + m + l exactly (h the upper half of x, m
// what is left rounded to bf16, l the rest, which bf16 holds; below 2^-109 its subnormals end and l is off by up to 2^-134).  Of the nine products of parts the six that count, h h, h m, m h, h l, m m and l h, go through
// mfma_f32_32x32x16_bf16, summed in 32 bits: what is left out is below 2^-22 of a product, less than such sums
// of 128 products round (three prompts of up to 1021 tokens: 4.1e-7 from the values in 64 bits, plain 32-bit products and sums 5.5e-7), and a sixth of the bf16 rate is 2.7 times the
// rate of mfma_f32_32x32x2, whose kernel took 4770 us for a prompt of 8000 tokens (8 heads of 4; 524 Gflop), this 2586: 203 Tflop/s, 1220 of bf16, which is
// where the library's products of such numbers end as well.  Bound by the matrix units, 96 products of 32 clocks for 32 keys and 32 rows of a wave, and short of workgroups below some
// 2000 tokens (1000: 110 us).
//
// Tiles of 32 keys come to LDS as they are, 1 KB blocks of two rows by the wave that then takes them apart and writes the parts, between the products of
// the tile before: one barrier a tile.  Parts lie as in attend_prompt.hip: four columns of 64 bytes a row.
// A tile that holds an infinity or NaN, whose parts would make NaN of infinities, is put together again and goes through the products of 32 bits; such, and tiles
// with a mask, stand outside the loop of whole tiles (in one loop with them, the sums were copied from path to path: 8000 tokens 4860 us).

#include <type_traits>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

typedef short s16x4a __attribute__((ext_vector_type(4)));

constexpr int kKeys = 32;              // of a tile
constexpr float kLoose = 8.f;          // (as in attend_prompt.hip)
constexpr int kPart = kKeys * 256;     // bytes of one part of a tile's keys or values

struct PromptF32Args {
    AttendCall c;
    float scale_log2;
    int groups, rows, row_tiles;
};

struct Parts {                         // of eight numbers
    u32x4a h, m, l;
};
// The parts of two numbers; `odd` becomes NaN where one is not finite.
__device__ __forceinline__ void apart(float x, float y, uint32_t& h, uint32_t& m, uint32_t& l, float& odd) {
    const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
    h = __builtin_amdgcn_perm(b, a, 0x07060302u);
    const float x1 = x - __uint_as_float(a & 0xFFFF0000u), y1 = y - __uint_as_float(b & 0xFFFF0000u);
    odd = __builtin_fmaf(x1, 0.f, odd);
    odd = __builtin_fmaf(y1, 0.f, odd);
    m = pack_bf16(x1, y1);
    l = pack_bf16(x1 - __uint_as_float(m << 16), y1 - __uint_as_float(m & 0xFFFF0000u));
}
__device__ __forceinline__ Parts apart(f32x4a x, f32x4a y, float& odd) {
    Parts p;
    uint32_t h[4], m[4], l[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        apart(x[2 * i], x[2 * i + 1], h[i], m[i], l[i], odd);
        apart(y[2 * i], y[2 * i + 1], h[2 + i], m[2 + i], l[2 + i], odd);
    }
    p.h = (u32x4a){h[0], h[1], h[2], h[3]};
    p.m = (u32x4a){m[0], m[1], m[2], m[3]};
    p.l = (u32x4a){l[0], l[1], l[2], l[3]};
    return p;
}
// Where a number is not finite: all of it in h (a NaN stays one), zeros in m and l.
__device__ __forceinline__ void keep_whole(Parts& p, f32x4a x, f32x4a y) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(i < 4 ? x[i] : y[i - 4]), low = i % 2 ? 0xFFFF0000u : 0x0000FFFFu;
        if ((a & 0x7F800000u) != 0x7F800000u) continue;
        if (a & 0x007FFFFFu) p.h[i / 2] |= i % 2 ? 0x00400000u : 0x00000040u;
        p.m[i / 2] &= ~low;
        p.l[i / 2] &= ~low;
    }
}
__device__ __forceinline__ float together(uint32_t h, uint32_t m, uint32_t l, bool upper) {
    const auto of = [&](uint32_t x) { return __uint_as_float(upper ? x & 0xFFFF0000u : x << 16); };
    return of(h) + (of(m) + of(l));
}

__device__ __forceinline__ f32x16a product(u32x4a x, u32x4a y, f32x16a z) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, x), __builtin_bit_cast(bf16x8a, y), z, 0, 0, 0);
}
__device__ __forceinline__ u32x2 read_transposed(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4a*)p));
}

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES / 4) void attend_prompt_f32_kernel(PromptF32Args a) {
    constexpr int kTileRows = WAVES * 32, kBlocks = 16 / WAVES, kEvery = 3 * WAVES / 4;
    __shared__ __attribute__((aligned(16))) char Ks[2][3 * kPart], Vs[2][3 * kPart], raw[2][kKeys * 512];
    __shared__ int not_finite[2];      // the last tile of either buffer with an infinity or NaN
    if (threadIdx.x < 2) not_finite[threadIdx.x] = -1;
    const AttendCall& c = a.c;
    const int g = blockIdx.x % a.groups, row_tile = a.row_tiles - 1 - blockIdx.x / a.groups;      // long ones first
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int b = g / c.kv, head = g % c.kv;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n;
    const int t_first = row_tile * kTileRows / c.group, t_last = min(c.m - 1, (row_tile * kTileRows + kTileRows - 1) / c.group);
    const Seen seen = seen_rows(length, c.m, t_first, t_last, c.window, c.sinks);
    const int first_tiles = (seen.first + kKeys - 1) / kKeys, tiles = first_tiles + (seen.high - seen.low + kKeys - 1) / kKeys;
    const auto row_of = [&](int tile) ALWAYS_INLINE { return tile < first_tiles ? tile * kKeys : seen.low + (tile - first_tiles) * kKeys; };
    const auto count_of = [&](int tile) ALWAYS_INLINE { return min(kKeys, (tile < first_tiles ? seen.first : seen.high) - row_of(tile)); };

    const int R0 = row_tile * kTileRows + wave * 32, R = min(R0 + col, a.rows - 1), t = R / c.group, p = length - c.m + t;
    const int p_first = length - c.m + min(R0, a.rows - 1) / c.group, p_last = length - c.m + min(R0 + 31, a.rows - 1) / c.group;
    const int64_t q_row = (((int64_t)b * c.m + t) * c.kv + head) * c.group + R % c.group;
    Parts q[8];                        // channels 16 i + 8 half + 0..7
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const f32x4a* from = (const f32x4a*)((const char*)c.Q + q_row * 512) + 4 * i + 2 * half;
        const f32x4a x = from[0], y = from[1];
        float odd = 0.f;
        q[i] = apart(x, y, odd);
        if (odd != odd) keep_whole(q[i], x, y);
    }

    const char* Kg = (const char*)c.K + (int64_t)g * c.stride * 512;
    const char* Vg = (const char*)c.V + (int64_t)g * c.stride * 512;
    const uint32_t raw_lds = lds_address(&raw[0][0]);
    const auto fetch = [&](int tile) ALWAYS_INLINE {
        const int64_t j0 = row_of(tile);
        const int count = count_of(tile);
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const int block = wave * kBlocks + i, row = block * 2 + half;
            const uint32_t from = min(row, count - 1) * 512 + (lane & 31) * 16;
            dma16(raw_lds + block * 1024, Kg + j0 * 512, from);
            dma16(raw_lds + kKeys * 512 + block * 1024, Vg + j0 * 512, from);
        }
    };
    // This wave's rows of a tile into parts: 32 pieces of eight channels a block, K's by lanes 0..31, V's by the others.  Block i; `odd` as above.
    // (eight lanes write 128 bytes side by side)
    const int piece_row = col >> 2 & 1, piece_at = (col & 3) + (col >> 3) * 4;
    struct Piece {
        f32x4a x, y;
        Parts z;
    };
    const auto read_piece = [&](Piece& e, int i) ALWAYS_INLINE {
        const f32x4a* from = (const f32x4a*)(raw[half] + (wave * kBlocks + i) * 1024 + piece_row * 512) + piece_at * 2;
        e.x = from[0], e.y = from[1];
    };
    const auto part_pair = [&](Piece& e, int j, float& odd) ALWAYS_INLINE {
        const f32x4a& x = j < 2 ? e.x : e.y;
        uint32_t h, m, l;
        apart(x[j % 2 * 2], x[j % 2 * 2 + 1], h, m, l, odd);
        e.z.h[j] = h, e.z.m[j] = m, e.z.l[j] = l;
    };
    const auto write_piece = [&](const Piece& e, int tile, int i) ALWAYS_INLINE {
        const int row = (wave * kBlocks + i) * 2 + piece_row;
        char* at = (half ? Vs[tile & 1] : Ks[tile & 1]) + (piece_at >> 2) * (kKeys * 64) + row * 64 + (((piece_at & 3) ^ (half ? 0 : (row >> 1) & 3)) << 4);
        *(u32x4a*)at = e.z.h;
        *(u32x4a*)(at + kPart) = e.z.m;
        *(u32x4a*)(at + 2 * kPart) = e.z.l;
    };
    const auto take_apart = [&](int tile, int i, float& odd, bool careful) ALWAYS_INLINE {
        Piece e;
        read_piece(e, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) part_pair(e, j, odd);
        if (careful) keep_whole(e.z, e.x, e.y);
        write_piece(e, tile, i);
    };
    const auto taken_apart = [&](int tile, float odd) ALWAYS_INLINE {
        if (odd == odd) return;
#pragma unroll 1
        for (int i = 0; i < kBlocks; ++i) take_apart(tile, i, odd, true);
        not_finite[tile & 1] = tile;
    };
    const auto take_all_apart = [&](int tile) ALWAYS_INLINE {
        float odd = 0.f;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) take_apart(tile, i, odd, false);
        taken_apart(tile, odd);
    };

    const int l16 = lane & 15, dhalf = (lane >> 4) & 1;
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    const int v_at = (4 * half + l16 / 4) * 64 + dhalf * 32 + (l16 & 3) * 8;

    f32x16a o[4];                      // o[db][i]: channel 32 db + 8 (i / 4) + 4 half + i % 4
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    // (-infinity and a guard below, not kNoScore: without the guard eight waves spill 551 registers, so 229: 8000 tokens 3690 us, so 2720)
    float top = -INFINITY, sum = 0.f;

    // Takes a tile's scores into the running softmax: s become the weights.
    const auto weigh = [&](auto masked, f32x16a& s, int far, int near, int sink) ALWAYS_INLINE {
        if (decltype(masked)::value)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = i / 4 * 8 + i % 4;
                s[i] = key <= far && (key > near || key < sink) ? s[i] : -INFINITY;
            }
        float most = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
        most = halves_max(most) * a.scale_log2;
        if (__any(most > top + kLoose)) {
            const float next = most > top + kLoose ? most : top, keep = next == top ? 1.f : __builtin_amdgcn_exp2f(top - next);
            sum *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db) o[db] *= keep;
            top = next;
        }
        const float off = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2, -off));
            sum += s[i];
        }
    };
    // Between the products of scores the next tile, where there is one, is taken apart.
    const auto take = [&](auto masked, int tile, bool more, int far, int near, int sink) ALWAYS_INLINE {
        const char *Kt = Ks[tile & 1], *Vt = Vs[tile & 1];
        f32x16a s, small;
        float odd = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f, small[i] = 0.f;
        Parts k[2];
        const auto load_keys = [&](int i) ALWAYS_INLINE {
            const char* at = Kt + k_at[i & 1] + (i >> 1) * (kKeys * 64);
            k[i & 1].h = *(const u32x4a*)at;
            k[i & 1].m = *(const u32x4a*)(at + kPart);
            k[i & 1].l = *(const u32x4a*)(at + 2 * kPart);
        };
        // Work between the products: a pair of the next tile's numbers after every third, its pieces read and written four pairs apart; the next step's keys.
        Piece piece[2];
        load_keys(0);
        read_piece(piece[0], 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Parts& x = k[i & 1];
#pragma unroll
            for (int j = 0; j < 6; ++j) {
                if (j == 0) s = product(x.h, q[i].h, s);
                if (j == 1) small = product(x.m, q[i].h, small);
                if (j == 2) s = product(x.h, q[i].m, s);
                if (j == 3) small = product(x.m, q[i].m, small);
                if (j == 4) s = product(x.h, q[i].l, s);
                if (j == 5) small = product(x.l, q[i].h, small);
                if (j == 0 && i < 7) load_keys(i + 1);
                const int n = i * 6 + j, pair = n / kEvery, e = pair / 4;
                if (n % kEvery == kEvery - 1 && e < kBlocks) {
                    part_pair(piece[e & 1], pair % 4, odd);           // (without a next tile, what the last one left)
                    if (pair % 4 == 0 && e + 1 < kBlocks) read_piece(piece[(e + 1) & 1], e + 1);
                    if (pair % 4 == 3) write_piece(piece[e & 1], tile + 1, e);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (more) {
            taken_apart(tile + 1, odd);
            if (tile + 2 < tiles) fetch(tile + 2);
        }
        Parts v[2][2];
        const auto load_values = [&](int j) ALWAYS_INLINE {                            // of 16 keys j / 2, channels 64 (j % 2) + 0..63
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const char* at = Vt + v_at + ((j & 1) * 2 + d) * (kKeys * 64) + (j >> 1) * 1024;
                u32x4a* to[3] = {&v[j & 1][d].h, &v[j & 1][d].m, &v[j & 1][d].l};
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    const u32x2 x = read_transposed(at + part * kPart), y = read_transposed(at + part * kPart + 512);
                    *to[part] = (u32x4a){x.x, x.y, y.x, y.y};
                }
            }
        };
        load_values(0);
        s += small;
        weigh(masked, s, far, near, sink);
        float unused = 0.f;
        Parts w[2];
        const auto weights = [&](int u) ALWAYS_INLINE {
            w[u] = apart((f32x4a){s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3]}, (f32x4a){s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]}, unused);
        };
        weights(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j < 3) load_values(j + 1);
            const Parts &y = w[j >> 1], &v0 = v[j & 1][0], &v1 = v[j & 1][1];
            f32x16a &o0 = o[(j & 1) * 2], &o1 = o[(j & 1) * 2 + 1];
            o0 = product(v0.l, y.h, o0);
            o1 = product(v1.l, y.h, o1);
            o0 = product(v0.m, y.m, o0);
            o1 = product(v1.m, y.m, o1);
            if (j == 0) weights(1);
            o0 = product(v0.h, y.l, o0);
            o1 = product(v1.h, y.l, o1);
            o0 = product(v0.m, y.h, o0);
            o1 = product(v1.m, y.h, o1);
            o0 = product(v0.h, y.m, o0);
            o1 = product(v1.h, y.m, o1);
            o0 = product(v0.h, y.h, o0);
            o1 = product(v1.h, y.h, o1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto take_whole_numbers = [&](int tile, int far, int near, int sink) ALWAYS_INLINE {
        const char *Kt = Ks[tile & 1], *Vt = Vs[tile & 1];
        f32x16a s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {                     // four channels of 32: half a piece
            const char* at = Kt + (i >> 2) * (kKeys * 64) + col * 64 + ((((i & 2) + half) ^ ((col >> 1) & 3)) << 4) + (i & 1) * 8;
            const u32x2 h = *(const u32x2*)at, m = *(const u32x2*)(at + kPart), l = *(const u32x2*)(at + 2 * kPart);
            const f32x4a x = ((const f32x4a*)((const char*)c.Q + q_row * 512))[(i >> 1) * 4 + half * 2 + (i & 1)];
#pragma unroll
            for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(together(h[j / 2], m[j / 2], l[j / 2], j % 2), x[j], s, 0, 0, 0);
        }
        weigh(std::true_type{}, s, far, near, sink);
        // An infinity or NaN must not meet the zero weight of a row that does not see it: a zero in its place, ..
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const char* at = Vt + db * (kKeys * 64) + (i / 4 * 8 + half * 4 + i % 4) * 64 + col * 2;
                const float v = together(*(const uint16_t*)at, *(const uint16_t*)(at + kPart), *(const uint16_t*)(at + 2 * kPart), false);
                o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32((__float_as_uint(v) & 0x7F800000u) == 0x7F800000u ? 0.f : v, s[i], o[db], 0, 0, 0);
            }
        }
        // .. and then they reach the rows that do see them: whatever the weight, an infinity or NaN comes of it.
        for (int key = 0; key < kKeys; ++key) {
            const int here = key - half * 4;
            if (!(here <= far && (here > near || here < sink))) continue;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x2 v = *(const u32x2*)(Vt + db * (kKeys * 64) + key * 64 + i * 16 + half * 8);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t x = w % 2 ? v[w / 2] & 0xFFFF0000u : v[w / 2] << 16;
                        if ((x & 0x7F800000u) == 0x7F800000u) o[db][4 * i + w] += __uint_as_float(x);
                    }
                }
        }
    };

    if (tiles > 0) {
        fetch(0);
        dma_wait();
    }
    __syncthreads();                   // (not_finite)
    if (tiles > 0) {
        take_all_apart(0);
        if (tiles > 1) fetch(1);
    }
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
        // tiles that all of this wave's tokens see all of, ..
        for (; tile < tiles; ++tile) {
            const int j0 = row_of(tile);
            if (!(count_of(tile) == kKeys && j0 + kKeys - 1 <= p_first && (c.window <= 0 || p_last - j0 < c.window || j0 + kKeys <= c.sinks))) break;
            if (__builtin_amdgcn_readfirstlane(not_finite[tile & 1]) == tile) break;
            dma_wait();
            take(std::false_type{}, tile, tile + 1 < tiles, 0, 0, 0);
            __syncthreads();
        }
        if (tile >= tiles) break;
        // .. and one of the others.  Keys of it that a row sees, counted from the half's first: near < key <= far, and those below `sink`.
        const int j0 = row_of(tile);
        const int far = min(p - j0, count_of(tile) - 1) - half * 4, near = (c.window > 0 ? p - j0 - c.window : -1) - half * 4, sink = c.sinks - j0 - half * 4;
        const bool none = j0 > p_last || (c.window > 0 && j0 + kKeys - 1 <= p_first - c.window && j0 >= c.sinks), odd = __builtin_amdgcn_readfirstlane(not_finite[tile & 1]) == tile;
        dma_wait();
        if (!none && !odd) {
            take(std::true_type{}, tile, tile + 1 < tiles, far, near, sink);
        } else {
            if (tile + 1 < tiles) {
                take_all_apart(tile + 1);
                if (tile + 2 < tiles) fetch(tile + 2);
            }
            if (!none) take_whole_numbers(tile, far, near, sink);
        }
        __syncthreads();
    }

    sum = halves_sum(sum);
    if (R0 + col >= a.rows) return;
    const bool empty = sum == 0.f;
    const float over = empty ? 0.f : 1.f / sum;
    char* out = (char*)c.out + q_row * 512;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x16a& x = o[db];
            *(f32x4a*)(out + (db * 32 + i * 8 + half * 4) * 4) = (f32x4a){x[4 * i] * over, x[4 * i + 1] * over, x[4 * i + 2] * over, x[4 * i + 3] * over};
        }
    if (c.lse && half == 0) c.lse[((int64_t)b * c.kv * c.group + head * c.group + R % c.group) * c.m + t] = empty ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

hipError_t launch_attend_prompt_f32(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream) {
    PromptF32Args a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.groups = (int)(call.count * call.kv);
    a.rows = call.m * call.group;
    const auto launch = [&](auto kernel, int waves) {
        a.row_tiles = (a.rows + waves * 32 - 1) / (waves * 32);
        kernel<<<(unsigned)((int64_t)a.groups * a.row_tiles), waves * 64, 0, stream>>>(a);
        return hipGetLastError();
    };
    // 256 rows a workgroup, two waves a SIMD, where whole ones give three for two units; 128 below.  8 heads' prompts, 256 and 128: 2400 tokens 388 and 344 us, 3200 528
    // and 584, 8000 2586 and 3204.
    if (2 * (int64_t)a.groups * (a.rows / 256) >= 3 * (int64_t)ctx->num_cu) return launch(attend_prompt_f32_kernel<8>, 8);
    return launch(attend_prompt_f32_kernel<4>, 4);
}

}  // namespace curdkv
