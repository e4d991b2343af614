// Attention of many tokens (prompts) over a bf16 cache: tiles of 64 keys against 32 rows R a wave, the softmax's maximum and sum running
// along.  Bound by the matrix units and the exponentials: 4 * 128 flops and one exponential for a visible (row, key).  Measured, on several cards: 8192 tokens of 32 heads (550
// Gflop) 530 to 562 us, 980 to 1040 Tflop/s; 32768 through windows of 4096 (2064 Gflop) 2040 to 2190 us, 940 to 1010 Tflop/s; a library product of 8192^3 reaches 1180 to 1240.  What holds
// it there is the power that the numbers' switching costs: zeros in place of random ones take 413 us, and the product 1780 Tflop/s.  (In a series of launches: after a pause the first dozen
// take up to a third longer, until the clock has settled.)
// Four waves of 32 rows: eight share a tile's loads (4096 tokens 164 us, so 154), but with windows, whose tiles have masks, wait for each other (500: 148, so 161); 64 rows
// a wave leave one wave a SIMD (973 Tflop/s, so 904).
//
// S^T = K Q^T by mfma_f32_32x32x16_bf16: a lane has the scores of one row R = lane % 32, for the keys 8 i + 4 (lane / 32) + 0..3 of 32,
// which is what the B operand of O^T = V^T P^T takes if the 16 keys of a product are counted in that order; P never leaves its
// registers.  The rows of all query heads of a KV head stand side by side (R = token * group + head), so that the tokens of a
// tile are few and little is computed beyond the diagonal.
// K and V tiles go from memory straight to LDS, two buffers each, as four columns of 64 bytes a row: what a wave's transposing read of V
// takes (8 keys, 32 channels) lies side by side; K's 16-byte pieces are permuted within a row's 64 bytes by (row / 2) % 4, so that eight rows' reads of the
// same piece meet different banks.
//
// The reference point of a row's exponentials is its maximum only to within 2^8: it moves, and what has been summed is scaled, when the
// maximum passes it by more, so that most tiles scale nothing.  Weights are then up to 2^8; in bf16 they are rounded by 2^-8 of themselves for their product with V, as
// weights up to 1 are, and their sum takes them in 32 bits.  Results lie 0.0022 of themselves from the values in 64 bits, 0.0016 with weights of 32 bits (the results' own rounding):
// weights in two parts would be half as many products again where products are the bound.

#include <algorithm>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

typedef uint16_t u16x2a __attribute__((ext_vector_type(2)));
typedef short s16x4a __attribute__((ext_vector_type(4)));

constexpr int kKeys = 64;              // of a tile
constexpr float kLoose = 8.f;
constexpr int kWaves = 4, kTileRows = kWaves * 32;        // rows R of a workgroup

struct PromptArgs {
    AttendCall c;
    float scale_log2;
    int groups, rows, row_tiles;
    int parts;                         // workgroups that share out the tiles of keys of one row tile
    float* part_o;                     // parts > 1: [parts][groups * row_tiles * 128][128], un-normalised
    f32x2a* part_ml;                   // the same of reference points and sums
};

__device__ __forceinline__ u32x2 read_transposed(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4a*)p));
}
__device__ __forceinline__ uint32_t max_halves(uint32_t x, uint32_t y) {      // of either 16 bits
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2a, x), __builtin_bit_cast(u16x2a, y)));
}

// KEPT: kept rows, which all tokens see, are the first tiles (there is no window then); the cache is the tokens since.
template <bool KEPT>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_prompt_kernel(PromptArgs a) {
    constexpr int kStage = 16 / kWaves;
    __shared__ __attribute__((aligned(16))) char Ks[2][kKeys * 256], Vs[2][kKeys * 256];
    __shared__ int not_finite;         // a tile whose V holds an infinity or NaN
    if (threadIdx.x == 0) not_finite = -1;
    const AttendCall& c = a.c;
    const int g = blockIdx.x % a.groups, part = blockIdx.x / a.groups % a.parts;
    const int row_tile = a.row_tiles - 1 - blockIdx.x / a.groups / a.parts;                        // long ones first
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int b = g / c.kv, head = g % c.kv;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n;

    const int t_first = row_tile * kTileRows / c.group, t_last = min(c.m - 1, (row_tile * kTileRows + kTileRows - 1) / c.group);
    const Seen seen = seen_rows(length, c.m, t_first, t_last, c.window, c.sinks);
    int64_t kept_begin = 0;
    int first = seen.first;
    if (KEPT) {
        const int64_t begin = min(max(c.offsets[g], (int64_t)0), c.total);
        first = __builtin_amdgcn_readfirstlane((int)(min(max(c.offsets[g + 1], begin), c.total) - begin));
        kept_begin = uniform(begin);
    }
    const int first_tiles = (first + kKeys - 1) / kKeys, tiles = first_tiles + (seen.high - seen.low + kKeys - 1) / kKeys;
    const int start = (int)((int64_t)tiles * part / a.parts), stop = (int)((int64_t)tiles * (part + 1) / a.parts);
    const auto row_of = [&](int tile) ALWAYS_INLINE { return tile < first_tiles ? tile * kKeys : seen.low + (tile - first_tiles) * kKeys; };
    const auto count_of = [&](int tile) ALWAYS_INLINE { return min(kKeys, (tile < first_tiles ? first : seen.high) - row_of(tile)); };

    // this lane's rows
    const int R0 = row_tile * kTileRows + wave * 32;
    const int R = min(R0 + col, a.rows - 1), t = R / c.group, p = length - c.m + t;
    const int64_t query_row = (((int64_t)b * c.m + t) * c.kv + head) * c.group + R % c.group;
    u32x4a q[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = ((const u32x4a*)((const char*)c.Q + query_row * 256))[2 * s + half];

    const char* Kg = (const char*)c.K + (int64_t)g * c.stride * 256;
    const char* Vg = (const char*)c.V + (int64_t)g * c.stride * 256;
    // A tile's 1 KB blocks of 16 rows' columns: this wave's share.
    const uint32_t k_lds = lds_address(&Ks[0][0]), v_lds = lds_address(&Vs[0][0]);
    const int d_row = lane >> 2, d_piece = lane & 3;
    const auto fetch = [&](uint32_t lds, const char* rows, const void* kept, int tile, bool keys) ALWAYS_INLINE {
        const char* from = rows + (int64_t)row_of(tile) * 256;
        uint32_t to = lds + (tile & 1) * (kKeys * 256) + wave * (kStage * 1024);
        if (KEPT) {
            if (tile < first_tiles) from = (const char*)kept + (kept_begin + tile * kKeys) * 256;
            from = (const char*)uniform((int64_t)from);
            to = __builtin_amdgcn_readfirstlane(to);
        }
        const int count = count_of(tile);
#pragma unroll
        for (int i = 0; i < kStage; ++i) {
            const int block = wave * kStage + i, column = block >> 2, row0 = (block & 3) * 16;
            const uint32_t row = min(row0 + d_row, count - 1) * 256 + column * 64, piece = keys ? d_piece ^ ((d_row >> 1) & 3) : d_piece;
            dma16(to + i * 1024, from, row + (piece << 4));
        }
    };
    const auto fetch_k = [&](int tile) ALWAYS_INLINE { fetch(k_lds, Kg, c.K_kept, tile, true); };
    const auto fetch_v = [&](int tile) ALWAYS_INLINE { fetch(v_lds, Vg, c.V_kept, tile, false); };

    // this lane's operands within a tile: K row col, piece 2 x + half; V rows 4 half + lane16 / 4 (+ 8), channels 32 db + ..
    const int l16 = lane & 15, dhalf = (lane >> 4) & 1;
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    const int v_at = (4 * half + l16 / 4) * 64 + dhalf * 32 + (l16 & 3) * 8;

    f32x16a o[4];
    float ref = kNoScore, sum = 0.f, top;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    const auto product = [](u32x4a x, u32x4a y, f32x16a z) ALWAYS_INLINE {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, x), __builtin_bit_cast(bf16x8a, y), z, 0, 0, 0);
    };
    const auto scores = [&](int tile, f32x16a (&x)[2]) ALWAYS_INLINE {
        const char* Kt = Ks[tile & 1];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kb][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const u32x4a k = *(const u32x4a*)(Kt + k_at[i & 1] + (i >> 1) * 4096 + kb * 2048);
                x[kb] = product(k, q[i], x[kb]);
            }
        }
    };
    // Keys of a tile that a row sees, counted from the half's first: near < key <= far, and those below `sink`.
    struct Range {
        int far, near, sink;
        __device__ __forceinline__ bool has(int key) const { return key <= far && (key > near || key < sink); }
    };
    const auto range_of = [&](int tile) ALWAYS_INLINE {
        if (KEPT && tile < first_tiles) return Range{count_of(tile) - 1 - half * 4, -5, 0};
        const int j0 = row_of(tile);
        return Range{min(p - j0, count_of(tile) - 1) - half * 4, (c.window > 0 ? p - j0 - c.window : -1) - half * 4, c.sinks - j0 - half * 4};
    };
    const auto top_of = [&](const f32x16a (&x)[2]) ALWAYS_INLINE {
        float y = x[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) y = fmaxf(y, x[kb][i]);
        return halves_max(y) * a.scale_log2;
    };
    const auto raise = [&]() ALWAYS_INLINE {
        if (__any(top > ref + kLoose)) {
            const float next = top > ref + kLoose ? top : ref;
            const float keep = next == ref ? 1.f : __builtin_amdgcn_exp2f(ref - next);
            sum *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db) o[db] *= keep;
            ref = next;
        }
    };
    // A tile that may hold rows that some token does not see.
    const auto masked_step = [&](int tile) ALWAYS_INLINE {
        f32x16a s[2];
        scores(tile, s);
        // Whether the tile of V holds an infinity or NaN: every wave looks at its share of it.
        const char* Vt = Vs[tile & 1];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 16 / kWaves; ++i) {
            const u32x4a x = *(const u32x4a*)(Vt + (wave * (16 / kWaves) + i) * 1024 + lane * 16);
#pragma unroll
            for (int w = 0; w < 4; ++w) most = max_halves(most, x[w] & 0x7FFF7FFFu);
        }
        if ((most & 0xFFFFu) >= 0x7F80u || most >= 0x7F800000u) not_finite = tile;
        __syncthreads();
        if (tile + 2 < stop) fetch_k(tile + 2);
        if (tile + 1 < stop) fetch_v(tile + 1);
        const Range r = range_of(tile);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = r.has(kb * 32 + i / 4 * 8 + i % 4) ? s[kb][i] : -INFINITY;
        top = top_of(s);
        raise();
        uint32_t pb[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 4][i & 15], a.scale_log2, -ref));
            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 4][(i & 15) + 1], a.scale_log2, -ref));
            sum += x + y;
            pb[i / 2] = pack_bf16(x, y);
        }
        const bool finite = __builtin_amdgcn_readfirstlane(not_finite) != tile;
        if (finite) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    const u32x2 x = read_transposed(Vt + v_at + db * 4096 + u * 1024), y = read_transposed(Vt + v_at + db * 4096 + u * 1024 + 512);
                    o[db] = product((u32x4a){x.x, x.y, y.x, y.y}, (u32x4a){pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]}, o[db]);
                }
        } else {
            // An infinity or NaN must not meet the zero weight of a row that does not see it: products with zeros in their place, ..
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    const u32x2 x = read_transposed(Vt + v_at + db * 4096 + u * 1024), y = read_transposed(Vt + v_at + db * 4096 + u * 1024 + 512);
                    u32x4a w = {x.x, x.y, y.x, y.y};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((w[e] & 0x7F80u) == 0x7F80u) w[e] &= 0xFFFF0000u;
                        if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] &= 0x0000FFFFu;
                    }
                    o[db] = product(w, (u32x4a){pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]}, o[db]);
                }
            // .. and then they reach the rows that do see them: whatever the weight, an infinity or NaN comes of it.
            const Range r = range_of(tile);
            for (int key = 0; key < kKeys; ++key) {
                if (!r.has(key - half * 4)) continue;
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // channels 32 db + 8 i + 4 half ..+3: half a piece
                        const u32x2 v = *(const u32x2*)(Vt + db * 4096 + key * 64 + i * 16 + half * 8);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t x = w % 2 ? v[w / 2] & 0xFFFF0000u : v[w / 2] << 16;
                            if ((x & 0x7F800000u) == 0x7F800000u) o[db][4 * i + w] += __uint_as_float(x);
                        }
                    }
            }
        }
        dma_wait();
        __syncthreads();
    };
    // Tiles begin .. end - 1, of which every token sees all: the next tile's 16 products with this one's exponentials between them, in the order
    // written (a matrix product every 7 other instructions keeps both pipes busy, and no more operands wait in registers than the next two products
    // need), then this one's 16 products with the next one's maximum.  `end` is a tile too (its scores are made, and dropped).
    const auto whole_steps = [&](int begin, int end) ALWAYS_INLINE {
        f32x16a s[2];
        scores(begin, s);
        top = top_of(s);
        __syncthreads();
        for (int tile = begin; tile < end; ++tile) {
            fetch_k(min(tile + 2, stop - 1));
            fetch_v(tile + 1);
            raise();
            const char *Kt = Ks[(tile + 1) & 1], *Vt = Vs[tile & 1];
            f32x16a next[2];
            uint32_t pb[16];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) next[kb][i] = 0.f;
            u32x4a k[2][2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) k[0][kb] = *(const u32x4a*)(Kt + k_at[0] + kb * 2048);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i < 7)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) k[(i + 1) & 1][kb] = *(const u32x4a*)(Kt + k_at[(i + 1) & 1] + ((i + 1) >> 1) * 4096 + kb * 2048);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) next[kb] = product(k[i & 1][kb], q[i], next[kb]);
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    const int kb = i >> 2, at = (i & 3) * 4 + j;
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][at], a.scale_log2, -ref));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][at + 1], a.scale_log2, -ref));
                    sum += x + y;
                    pb[kb * 8 + at / 2] = pack_bf16(x, y);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            u32x2 v[2][4][2];
            const auto values = [&](int u) ALWAYS_INLINE {
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int x = 0; x < 2; ++x) v[u & 1][db][x] = read_transposed(Vt + v_at + db * 4096 + u * 1024 + x * 512);
            };
            values(0);
            float most = next[0][0];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (u < 3) values(u + 1);
                const u32x4a pu = {pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]};
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    const u32x4a w = {v[u & 1][db][0].x, v[u & 1][db][0].y, v[u & 1][db][1].x, v[u & 1][db][1].y};
                    o[db] = product(w, pu, o[db]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, next[u >> 1][(u & 1) * 8 + i]);
                __builtin_amdgcn_sched_barrier(0);
            }
            top = halves_max(most) * a.scale_log2;
            s[0] = next[0];
            s[1] = next[1];
            dma_wait();
            __syncthreads();
        }
    };

    if (start < stop) {
        fetch_k(start);
        fetch_v(start);
        if (start + 1 < stop) fetch_k(start + 1);
        dma_wait();
        __syncthreads();
        const int whole_end = min(first_tiles + max(0, (min(seen.high, seen.p0 + 1) - seen.low) / kKeys), stop - 1);
        const int hidden = c.window > 0 ? max(0, seen.p1 - c.window + 1 - seen.low) : 0;         // rows from `low` on that the last token does not see
        const int whole_begin = max(min(first_tiles + (hidden + kKeys - 1) / kKeys, whole_end), start);
        int tile = start;
        if (KEPT && tile < min(first / kKeys, stop - 1)) {
            whole_steps(tile, min(first / kKeys, stop - 1));
            tile = min(first / kKeys, stop - 1);
        }
        for (int turn = 0; turn < 2; ++turn) {             // masked tiles, whole ones, masked ones
            const int end = turn == 0 ? whole_begin : stop;
            for (; tile < end; ++tile) masked_step(tile);
            if (turn == 0 && tile < whole_end) {
                whole_steps(tile, whole_end);
                tile = whole_end;
            }
        }
    }

    const float total = halves_sum(sum);
    if (R0 + col >= a.rows) return;
    if (a.parts > 1) {
        const int64_t at = ((int64_t)part * a.groups + g) * a.row_tiles * kTileRows + R;
        float* to = a.part_o + at * 128 + half * 4;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x16a& x = o[db];
                *(f32x4a*)(to + db * 32 + i * 8) = (f32x4a){x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
            }
        if (half == 0) a.part_ml[at] = (f32x2a){ref, total};
        return;
    }
    const bool empty = total == 0.f;
    const float over = empty ? 0.f : 1.f / total;
    char* out = (char*)c.out + query_row * 256;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x16a& x = o[db];
            *(u32x2*)(out + (db * 32 + i * 8 + half * 4) * 2) =
                (u32x2){pack_bf16(x[4 * i] * over, x[4 * i + 1] * over), pack_bf16(x[4 * i + 2] * over, x[4 * i + 3] * over)};
        }
    if (c.lse && half == 0)
        c.lse[((int64_t)b * c.kv * c.group + head * c.group + R % c.group) * c.m + t] = empty ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * kLn2;
}

// Joins the parts of four rows, a wave a row, two channels a lane.
__global__ __launch_bounds__(256) void attend_prompt_join_kernel(PromptArgs a) {
    const AttendCall& c = a.c;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, g = (int)(at / a.rows), R = (int)(at - (int64_t)g * a.rows);
    if (g >= a.groups) return;
    const int64_t first = (int64_t)g * a.row_tiles * kTileRows + R, step = (int64_t)a.groups * a.row_tiles * kTileRows;
    float ref = kNoScore, sum = 0.f;
    for (int k = 0; k < a.parts; ++k) ref = fmaxf(ref, a.part_ml[first + k * step].x);
    f32x2a o = {0, 0};
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) {
        const f32x2a ml = a.part_ml[first + k * step], x = *(const f32x2a*)(a.part_o + (first + k * step) * 128 + lane * 2);
        const float weight = __builtin_amdgcn_exp2f(ml.x - ref);
        sum += weight * ml.y;
        o.x += weight * x.x;
        o.y += weight * x.y;
    }
    const bool empty = sum == 0.f;
    const float over = empty ? 0.f : 1.f / sum;
    const int b = g / c.kv, t = R / c.group, h = (g - b * c.kv) * c.group + R % c.group;
    ((uint32_t*)c.out)[(((int64_t)b * c.m + t) * c.kv * c.group + h) * 64 + lane] = pack_bf16(o.x * over, o.y * over);
    if (c.lse && lane == 0) c.lse[((int64_t)b * c.kv * c.group + h) * c.m + t] = empty ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

hipError_t launch_attend_prompt(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream) {
    PromptArgs a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.groups = (int)(call.count * call.kv);
    a.rows = call.m * call.group;
    a.row_tiles = (a.rows + kTileRows - 1) / kTileRows;
    // Few new tokens over a long cache: the tiles of keys shared out until every unit has two workgroups, 8 tiles each at least, as far as there is scratch.
    const int64_t blocks = (int64_t)a.groups * a.row_tiles, tiles = ((call.window > 0 ? std::min((int64_t)call.n, (int64_t)call.window + call.sinks + call.m) : call.n) + call.rows / a.groups) / kKeys;
    const int64_t part_bytes = blocks * kTileRows * (int64_t)(128 * sizeof(float) + sizeof(f32x2a)), room = call.scratch ? call.scratch_bytes - kScratchCounters : 0;
    int64_t parts = std::min(std::min(2 * ctx->num_cu / blocks, tiles / 8), room / part_bytes);
    // Two parts, which fill what one workgroup a unit leaves idle, take longer than one over short caches, and a join: 8 heads of 4, 768 new tokens (192 workgroups) over 3000 rows one
    // part 59 us, two 62, over 4000 74 and 72, 6000 108 and 98; 1024 (256) over 2000 43 and 54, 6000 111 and 112, 16000 283 and 260.  (Kept rows: heads are uneven, and parts of them
    // less so: 1024 tokens over 500 to 3276 of them 113 and 113, 4 sequences of 256 196 and 158.)
    if (parts == 2 && !call.offsets && 2 * tiles < blocks - 70) parts = 1;
    a.parts = parts > 1 ? (int)parts : 1;
    a.part_o = (float*)((char*)call.scratch + kScratchCounters);
    a.part_ml = (f32x2a*)(a.part_o + a.parts * blocks * kTileRows * 128);
    if (call.offsets) attend_prompt_kernel<true><<<(unsigned)(blocks * a.parts), kWaves * 64, 0, stream>>>(a);
    else attend_prompt_kernel<false><<<(unsigned)(blocks * a.parts), kWaves * 64, 0, stream>>>(a);
    if (a.parts > 1) attend_prompt_join_kernel<<<(unsigned)(((int64_t)a.groups * a.rows + 3) / 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace curdkv
