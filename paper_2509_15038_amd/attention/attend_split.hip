// Attention of a few tokens over long caches: the rows of a KV head are shared out over workgroups, of which the last one to be done joins the parts.
// out = softmax(q k / sqrt(d)) v with the running maximum M and sum L of a softmax: of two parts of the keys
// with (M1, L1, o1) and (M2, L2, o2), o un-normalised, the whole has M = max, L = L1 2^(M1-M) + L2 2^(M2-M) and o likewise
// (scores in units of log 2 throughout; all of it in 32 bits, but for the weights of bf16 rows, which their product with V takes in bf16 and their sum in 32).
//
// HBM-bound: every cache row is read once, by one wave, straight into the operand registers; nothing of the cache passes LDS.
// S^T = K Q^T: the rows of 16 keys are the A operand of mfma_f32_16x16x32_bf16 (16x16x4 for fp32), the 16 rows R of the queries
// the B operand, so that a lane holds scores of one R for the keys of its quarter of the wave.  Which key a row of the A operand
// stands for is free: they are picked so that a lane's scores are of T/4 consecutive keys, exactly what the B operand of
// O^T = V^T P^T wants of its lane, and P never leaves its registers.  V rows are loaded whole, 16 lanes of 8 channels a row,
// a lane holding the same 8 channels of the T/4 keys of its quarter; v_perm pairs them up into the A operand of eight products,
// product i for channels 8 eight_of(c) + i.
//
// Measured: a token over 131072 rows of 8 heads (537 MB) 91 us, 5.9 TB/s; of 32 sequences through windows of 4096 (404 MB) 66 us, 6.1 TB/s; 4 tokens of 8 sequences over
// 6553 kept rows a head (217 MB) 50 us, 4.3 TB/s; 32 sequences over 13107 kept rows a head in 4 bits (490 MB with their tails) 105 us, 4.7 TB/s: the heads' ends inside the shares
// (3 us each) and the join (4 us).  One sequence over 3276 kept rows a head 13 us: a chain of latencies, of which reading is 3.
// In fp32: the token over 131072 rows (1074 MB) 171 us, 6.3 TB/s; 32 sequences through windows of 4096 (808 MB) 156 us, 5.2 TB/s; the 4 tokens of 8 sequences (434 MB) 83 us, 5.2 TB/s; the 32
// sequences over rows in 4 bits 306 us, 1.7 TB/s.
// A workgroup of four waves a unit, each with two tiles of 16 keys (32 KB) in flight: more workgroups only add to what there is to join (launch_attend_split).
// A wave's next tile is asked for without a branch: in front of one the compiler waits for all that is in flight.

#include <algorithm>
#include <climits>
#include <cmath>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

typedef short s16x4a __attribute__((ext_vector_type(4)));

constexpr int kSplitWaves = 4;
constexpr int kRowTile = 16;           // rows R a workgroup handles
constexpr int kCounters = kScratchCounters / sizeof(int);      // items at most that share workgroups
constexpr int64_t kPartBytes = 128 * sizeof(float) + 2 * sizeof(float);     // of a row of partial results

struct SplitArgs {
    AttendCall c;
    float scale_log2;
    int items, rows, row_tiles;        // heads times tiles of their rows R; m * group; tiles of them
    int shares;                        // workgroups that share all items; every item is one's of its own where that is 0
    bool whole;                        // every item has workgroups of its own, as long as the shares are few tiles
    int least;                         // tiles of an item, on average, from which it pays to share it (3/8 of them in workgroups of its own)
    float weight;                      // parts of an item squared over its tiles, where reading and joining are in balance
    int* arrived;                      // [items]: workgroups that are done with their part of an item; 0 between the calls
    float* part_o;                     // [slots][16][128]: of workgroup w and item i at w + i, which no other pair has
    f32x2a* part_ml;                   // the same of maxima and sums
};

enum Format { kNone = -1, kBf16 = 0, kF32 = 1, kMxBf16 = 2, kMxF32 = 3 };

struct Queries {                       // the B operands of S^T for one lane
    u32x4a q[8];                       // 4 of bf16, or 32 floats
};

// Codes of 4 bits to two bf16 / floats; SEL: which byte
template <int SEL>
__device__ __forceinline__ uint32_t two_bf16(uint32_t codes, float unit) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, SEL));
}
template <int SEL>
__device__ __forceinline__ f32x2a two_f32(uint32_t codes, float unit) {
    return __builtin_bit_cast(f32x2a, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, SEL));
}
// A block's power of two, of which the conversions take the exponent alone: 0 is 2^-127, 255 makes NaN of every code.
__device__ __forceinline__ float unit_of(uint32_t scale) { return __uint_as_float(scale << 23); }

// A lane's part of the running softmax: column R = lane % 16, channels 8 eight_of(4 (lane / 16) + j) + i in o[i][j].
struct Running {
    f32x4a o[8];
    float top, sum;                    // of R so far (top: of all quarters; sum: of the lane's keys)
};

// o += V^T P^T for bf16 rows: v[e] the lane's 8 channels of key e of its quarter, p[e] that key's weights; of 16 keys, or of 32.  The weights are rounded to bf16 for it, as the
// prompts' are: results lie 0.0017 to 0.0019 of themselves from the values in 64 bits, 0.0016 to 0.0017 with weights of 32 bits, so nearly all of it is the results' own rounding.
__device__ __forceinline__ f32x4a product(u32x4a x, u32x4a y, f32x4a z) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8a, x), __builtin_bit_cast(bf16x8a, y), z, 0, 0, 0);
}
__device__ __forceinline__ f32x4a product(u32x2 x, u32x2 y, f32x4a z) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4a, x), __builtin_bit_cast(s16x4a, y), z, 0, 0, 0);
}
template <int E> struct PairsOf;       // E keys of a lane, two to a register
template <> struct PairsOf<4> { typedef u32x2 type; };
template <> struct PairsOf<8> { typedef u32x4a type; };
template <int E>
__device__ __forceinline__ void add_values(const u32x4a (&v)[E], const float* p, f32x4a* o) {
    typename PairsOf<E>::type pb, even, odd;
#pragma unroll
    for (int u = 0; u < E / 2; ++u) pb[u] = pack_bf16(p[2 * u], p[2 * u + 1]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
#pragma unroll
        for (int u = 0; u < E / 2; ++u) {
            even[u] = __builtin_amdgcn_perm(v[2 * u + 1][w], v[2 * u][w], 0x05040100u);
            odd[u] = __builtin_amdgcn_perm(v[2 * u + 1][w], v[2 * u][w], 0x07060302u);
        }
        o[2 * w] = product(even, pb, o[2 * w]);
        o[2 * w + 1] = product(odd, pb, o[2 * w + 1]);
    }
}
// (fp32 products: exact to 2^-24 a product, 1/16 of the bf16 rate, which the bytes of fp32 rows still hide; 4-bit rows under fp32 are bound by it: 64 products of 32 clocks for 16 keys of
// 2176 bytes are 2.6 TB/s at most)
__device__ __forceinline__ void add_values(const float (&v)[4][8], const float* p, f32x4a* o) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][i], p[e], o[i], 0, 0, 0);
}

// Infinities and NaN in rows that some R does not see must not meet its zero weight.  Zeros take their place, and the R that do see one
// (seen: a bit for each of the lane's keys) get it whatever its weight: where a product of "is such a value" with "is seen" is not zero.
constexpr uint32_t kInf16 = 0x7F80u;
template <int E>
__device__ __forceinline__ bool any_not_finite(const u32x4a (&v)[E]) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) bad |= (v[e][w] & kInf16) == kInf16 || (v[e][w] & (kInf16 << 16)) == kInf16 << 16;
    return __any(bad);
}
__device__ __forceinline__ bool any_not_finite(const float (&v)[4][8]) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i) bad |= (__float_as_uint(v[e][i]) & 0x7F800000u) == 0x7F800000u;
    return __any(bad);
}
__device__ __forceinline__ uint32_t kind_of(uint32_t x, uint32_t inf, uint32_t sign) {      // 0: +inf, 1: -inf, 2: NaN, 3: finite
    return (x & inf) != inf ? 3u : x == inf ? 0u : x == (inf | sign) ? 1u : 2u;
}
template <int E>
__device__ __forceinline__ void spread_not_finite(u32x4a (&v)[E], uint32_t seen, f32x4a* o) {
    typename PairsOf<E>::type sees, has;
#pragma unroll
    for (int u = 0; u < E / 2; ++u) sees[u] = (seen >> (2 * u) & 1 ? 0x3F80u : 0u) | (seen >> (2 * u + 1) & 1 ? 0x3F800000u : 0u);
#pragma unroll 1
    for (uint32_t kind = 0; kind < 3; ++kind) {
        const float value = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int u = 0; u < E / 2; ++u) {
                    const uint32_t x = v[2 * u][w] >> (16 * h) & 0xFFFFu, y = v[2 * u + 1][w] >> (16 * h) & 0xFFFFu;
                    has[u] = (kind_of(x, kInf16, 0x8000u) == kind ? 0x3F80u : 0u) | (kind_of(y, kInf16, 0x8000u) == kind ? 0x3F800000u : 0u);
                }
                const f32x4a z = product(has, sees, (f32x4a){0, 0, 0, 0});
#pragma unroll
                for (int j = 0; j < 4; ++j) o[2 * w + h][j] += z[j] > 0.f ? value : 0.f;
            }
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if ((v[e][w] & kInf16) == kInf16) v[e][w] &= 0xFFFF0000u;
            if ((v[e][w] & (kInf16 << 16)) == kInf16 << 16) v[e][w] &= 0xFFFFu;
        }
}
__device__ __forceinline__ void spread_not_finite(float (&v)[4][8], uint32_t seen, f32x4a* o) {
#pragma unroll 1
    for (uint32_t kind = 0; kind < 3; ++kind) {
        const float value = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f32x4a z = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                z = __builtin_amdgcn_mfma_f32_16x16x4f32(kind_of(__float_as_uint(v[e][i]), 0x7F800000u, 0x80000000u) == kind ? 1.f : 0.f, seen >> e & 1 ? 1.f : 0.f, z, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] += z[j] > 0.f ? value : 0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((__float_as_uint(v[e][i]) & 0x7F800000u) == 0x7F800000u) v[e][i] = 0.f;
}
template <class V>
__device__ __forceinline__ void add_values_masked(V& v, const float* p, uint32_t seen, f32x4a* o) {
    if (any_not_finite(v)) spread_not_finite(v, seen, o);
    add_values(v, p, o);
}

// Which eight channels a lane c of 16 has of a row of V: those of 4 bits come in whole lines of two rows (below).
__device__ __forceinline__ int eight_of(int c) { return (c & 7) * 2 + (c >> 3); }

// One tile of T keys in registers.  `first`: row of its first key in K and V; `count`: keys of it that there are (>= 1), the last
// one stands in for those beyond.  on = 0: nothing is asked of the tile, and all lanes load from its first bytes (the loads are there all the
// same: a branch around them would make the compiler wait for all that are in flight).  MASKED: some key of it is hidden from some R.
template <int F> struct Tile;

// K in whole lines of 128 bytes (a line that passes the caches in halves is fetched twice): an instruction takes 8 rows' 8 pieces of 16 bytes, lane
// (quarter, c) piece quarter + 4 (c / 8) of row c % 8 of 8.  What the A operand has in lane c < 8 from the second row of 8 and in lane c >= 8 from the
// first then lies 8 lanes off: x, of rows 0..7, and y, of rows 8..15, become pieces quarter and quarter + 4 of row c.
__device__ __forceinline__ void to_rows(u32x4a& x, u32x4a& y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a = (int)x[i], b = (int)y[i];
        x[i] = (uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x128, 0xF, 0xC, false);       // row_ror:8, lanes 8..15 of 16
        y[i] = (uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x128, 0xF, 0x3, false);       // lanes 0..7
    }
}

// Rows used once by a call that reads more than the caches hold pass them by.
template <bool PAST, class T>
__device__ __forceinline__ T fetched(const void* p) {
    return PAST ? __builtin_nontemporal_load((const T*)p) : *(const T*)p;
}

template <>
struct Tile<kBf16> {
    static constexpr int T = 16;
    u32x4a k[4], v[4];
    template <bool PAST>
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t*, const uint8_t*, int64_t first, int count, int lane, uint32_t on = ~0u) {
        const int c = lane & 15, quarter = lane >> 4;
        const char* Kb = (const char*)K + first * 256;
        const char* Vb = (const char*)V + first * 256;
        if (count == T) {
            const uint32_t k_at = ((c & 7) * 256 + (quarter + (c >> 3) * 4) * 16) & on;
#pragma unroll
            for (int s = 0; s < 4; ++s) k[s] = fetched<PAST, u32x4a>(Kb + k_at + (s & 1) * 2048 + (s >> 1) * 128);
            const uint32_t v_at = (quarter * 1024 + eight_of(c) * 16) & on;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fetched<PAST, u32x4a>(Vb + v_at + e * 256);
            return;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) k[s] = *(const u32x4a*)(Kb + (uint32_t)(min((s & 1) * 8 + (c & 7), count - 1) * 256 + (quarter + (c >> 3) * 4) * 16 + (s >> 1) * 128));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *(const u32x4a*)(Vb + (uint32_t)(min(quarter * 4 + e, count - 1) * 256 + eight_of(c) * 16));
    }
    __device__ __forceinline__ static void queries(Queries& q, const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 4; ++s) q.q[s] = ((const u32x4a*)row)[s * 4 + quarter];
    }
    __device__ __forceinline__ void scores(const Queries& q, float* s) {
        to_rows(k[0], k[1]);
        to_rows(k[2], k[3]);
        f32x4a a = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) a = product(k[i], q.q[i], a);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = a[j];
    }
    template <bool MASKED>
    __device__ __forceinline__ void values(const float* p, uint32_t seen, f32x4a* o) {
        if (MASKED) add_values_masked(v, p, seen, o);
        else add_values(v, p, o);
    }
};

template <>
struct Tile<kF32> {
    static constexpr int T = 16;
    u32x4a k[8];
    float v[4][8];
    template <bool PAST>
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t*, const uint8_t*, int64_t first, int count, int lane, uint32_t on = ~0u) {
        const int c = lane & 15, quarter = lane >> 4;
        const char* Kb = (const char*)K + first * 512;
        const char* Vb = (const char*)V + first * 512;
        if (count == T) {
            const uint32_t k_at = ((c & 7) * 512 + (quarter + (c >> 3) * 4) * 16) & on;
#pragma unroll
            for (int s = 0; s < 8; ++s) k[s] = fetched<PAST, u32x4a>(Kb + k_at + (s & 1) * 4096 + (s >> 1) * 128);
            const uint32_t v_at = (quarter * 2048 + eight_of(c) * 32) & on;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                *(f32x4a*)&v[e][0] = fetched<PAST, f32x4a>(Vb + v_at + e * 512);
                *(f32x4a*)&v[e][4] = fetched<PAST, f32x4a>(Vb + v_at + e * 512 + 16);
            }
            return;
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) k[s] = *(const u32x4a*)(Kb + (uint32_t)(min((s & 1) * 8 + (c & 7), count - 1) * 512 + (quarter + (c >> 3) * 4) * 16 + (s >> 1) * 128));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const char* row = Vb + (uint32_t)(min(quarter * 4 + e, count - 1) * 512 + eight_of(c) * 32);
            *(f32x4a*)&v[e][0] = *(const f32x4a*)row;
            *(f32x4a*)&v[e][4] = *(const f32x4a*)(row + 16);
        }
    }
    __device__ __forceinline__ static void queries(Queries& q, const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 8; ++s) q.q[s] = ((const u32x4a*)row)[s * 4 + quarter];
    }
    __device__ __forceinline__ void scores(const Queries& q, float* s) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) to_rows(k[i], k[i + 1]);
        f32x4a a = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i][j]), __uint_as_float(q.q[i][j]), a, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = a[j];
    }
    template <bool MASKED>
    __device__ __forceinline__ void values(const float* p, uint32_t seen, f32x4a* o) {
        if (MASKED) add_values_masked(v, p, seen, o);
        else add_values(v, p, o);
    }
};

// Rows in 4 bits: 64 bytes of codes (channel 2 i in the low half of byte i) and 4 scales, a power of two for 32 channels each.
// K: a lane's 16 bytes are one block of its key; V: 4 bytes of 8 channels of each key.
template <>
struct Tile<kMxBf16> {
    static constexpr int T = 32;
    u32x4a k[2], vs[2];
    uint32_t v[8], ks[2];
    template <bool PAST>
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t* Ks, const uint8_t* Vs, int64_t first, int count, int lane, uint32_t on = ~0u) {
        const int c = lane & 15, quarter = lane >> 4;
        const char* Kb = (const char*)K + first * 64;
        const char* Vb = (const char*)V + first * 64;
        const uint8_t* Kc = Ks + first * 4;
        const uint8_t* Vc = Vs + first * 4;
        if (count == T) {
            const uint32_t key = (c >> 2) * 8 + (c & 3), k_at = (key * 64 + quarter * 16) & on, v_at = (quarter * 512 + (c >> 3) * 64 + (c & 7) * 8) & on, ks_at = (key * 4 + quarter) & on;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                k[t] = fetched<PAST, u32x4a>(Kb + k_at + t * 256);
                ks[t] = *(Kc + ks_at + t * 16);
                __builtin_memcpy(&vs[t], Vc + quarter * 32 + t * 16, 16);       // (rows' scales lie at multiples of 4 bytes)
            }
            // (lanes c < 8 16 channels of the first of two rows, the others of the second: whole lines; values() makes 8 channels of both rows of it)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const u32x2 x = fetched<PAST, u32x2>(Vb + v_at + e * 64);
                v[e] = x.x, v[e + 1] = x.y;
            }
            return;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = min((c >> 2) * 8 + t * 4 + (c & 3), count - 1);
            k[t] = *(const u32x4a*)(Kb + (uint32_t)(key * 64 + quarter * 16));
            ks[t] = Kc[(uint32_t)(key * 4 + quarter)];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int key = min(quarter * 8 + e, count - 1), row = min(quarter * 8 + (e & ~1) + (c >> 3), count - 1);
            v[e] = *(const uint32_t*)(Vb + (uint32_t)(row * 64 + (c & 7) * 8 + (e & 1) * 4));
            vs[e / 4][e % 4] = *(const uint32_t*)(Vc + (uint32_t)(key * 4));
        }
    }
    __device__ __forceinline__ static void queries(Queries& q, const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 4; ++s) q.q[s] = ((const u32x4a*)row)[quarter * 4 + s];
    }
    __device__ __forceinline__ void scores(const Queries& q, float* s) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float unit = unit_of(ks[t]);
            f32x4a a = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a = product((u32x4a){two_bf16<0>(k[t][i], unit), two_bf16<1>(k[t][i], unit), two_bf16<2>(k[t][i], unit), two_bf16<3>(k[t][i], unit)}, q.q[i], a);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[t * 4 + j] = a[j];
        }
    }
    template <bool MASKED>
    __device__ __forceinline__ void values(const float* p, uint32_t seen, f32x4a* o) {
        const int shift = (threadIdx.x >> 1 & 3) * 8;                          // (of the block that the lane's channels lie in, eight_of(c) / 4)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {                                        // (lane c's second dword against lane c ^ 8's first)
            const int x = (int)v[e], y = (int)v[e + 1];
            v[e] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, 0x128, 0xF, 0xC, false);
            v[e + 1] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, 0x128, 0xF, 0x3, false);
        }
        u32x4a x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float unit = unit_of(vs[e / 4][e % 4] >> shift & 255u);
            x[e] = (u32x4a){two_bf16<0>(v[e], unit), two_bf16<1>(v[e], unit), two_bf16<2>(v[e], unit), two_bf16<3>(v[e], unit)};
        }
        // (a masked tile of kept rows ends them: its other keys repeat the last one, which every R sees, so nothing hidden is not finite alone)
        add_values(x, p, o);
    }
};

template <>
struct Tile<kMxF32> {
    static constexpr int T = 16;
    u32x4a k;
    uint32_t v[4], ks, vs[4];
    template <bool PAST>
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t* Ks, const uint8_t* Vs, int64_t first, int count, int lane, uint32_t on = ~0u) {
        const int c = lane & 15, quarter = lane >> 4;
        const int key = min(c, count - 1);
        k = *(const u32x4a*)((const char*)K + first * 64 + (uint32_t)(key * 64 + quarter * 16));
        ks = (Ks + first * 4)[(uint32_t)(key * 4 + quarter)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = min(quarter * 4 + e, count - 1);
            v[e] = *(const uint32_t*)((const char*)V + first * 64 + (uint32_t)(row * 64 + eight_of(c) * 4));
            vs[e] = (Vs + first * 4)[(uint32_t)(row * 4 + (eight_of(c) >> 2))];
        }
    }
    __device__ __forceinline__ static void queries(Queries& q, const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 8; ++s) q.q[s] = ((const u32x4a*)row)[quarter * 8 + s];
    }
    __device__ __forceinline__ static void wide(uint32_t codes, float unit, float* x) {
        *(f32x2a*)(x + 0) = two_f32<0>(codes, unit);
        *(f32x2a*)(x + 2) = two_f32<1>(codes, unit);
        *(f32x2a*)(x + 4) = two_f32<2>(codes, unit);
        *(f32x2a*)(x + 6) = two_f32<3>(codes, unit);
    }
    __device__ __forceinline__ void scores(const Queries& q, float* s) const {
        const float unit = unit_of(ks);
        f32x4a a = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[8];
            wide(k[i], unit, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) a = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], __uint_as_float(q.q[2 * i + j / 4][j % 4]), a, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = a[j];
    }
    template <bool MASKED>
    __device__ __forceinline__ void values(const float* p, uint32_t seen, f32x4a* o) {
        float x[4][8];
#pragma unroll
        for (int e = 0; e < 4; ++e) wide(v[e], unit_of(vs[e]), x[e]);
        add_values(x, p, o);
    }
};

// Takes a tile's scores into the running softmax.  MASKED: of the tile's keys, R sees those with a bit in `seen`.
template <int F, bool MASKED>
__device__ __forceinline__ void take(Running& r, Tile<F>& x, const Queries& q, float scale_log2, uint32_t seen) {
    constexpr int E = Tile<F>::T / 4;
    float s[E];
    x.scores(q, s);
    if (MASKED)
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] = seen >> e & 1 ? s[e] : -INFINITY;
    float top = s[0];
#pragma unroll
    for (int e = 1; e < E; ++e) top = fmaxf(top, s[e]);
    top = fmaxf(r.top, quarters_max(top) * scale_log2);
    if (__any(top > r.top)) {
        const float keep = top > r.top ? __builtin_amdgcn_exp2f(r.top - top) : 1.f;       // (0 before the first key)
        r.sum *= keep;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.o[i] *= keep;
        r.top = top;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale_log2, -r.top));
        r.sum += s[e];
    }
    x.template values<MASKED>(s, seen, r.o);
}

// What an item (a head's row tile) has to read: tiles that all its R see all of, from the kept rows, the first rows and the rows near; and
// tiles to be masked: the ends of those three, and where the window's edge and the diagonal pass.
struct Head {                          // what a head has, from the call's arrays
    int64_t begin;                     // first kept row
    int kept, length;                  // kept rows; rows of the cache
};
__device__ __forceinline__ Head head_of(const SplitArgs& a, int g) {
    const AttendCall& c = a.c;
    Head h{0, 0, 0};
    if (c.offsets) {
        h.begin = min(max(c.offsets[g], (int64_t)0), c.total);
        h.kept = (int)(min(max(c.offsets[g + 1], h.begin), c.total) - h.begin);
    }
    h.length = c.n > 0 ? (c.lengths ? min(max(c.lengths[g / c.kv], 0), c.n) : c.n) : 0;
    return h;
}
template <int FA, int FB>
struct Work {
    static constexpr int TA = Tile<FA == kNone ? kBf16 : FA>::T, TB = Tile<FB>::T;
    // What a tile costs, in units that the work is shared out by: its bytes, and the expansion of 4 bits.
    static constexpr int kUnitA = 1, kUnitB = FA == kMxF32 ? 3 : FA == kMxBf16 ? 2 : 1;
    int64_t begin = 0;                                     // first kept row
    int kept = 0, kept_tiles = 0;                          // (a head's rows are below 2^31, an item's units below 2^28)
    Seen seen;
    int t0, t1;
    int first_tiles, near_begin, near_end, near_tiles;     // whole first rows; of the tiles from seen.low on: whole ones, and all
    int cache_tiles;                                       // whole ones of the cache
    int low_masked, cache_masked;                          // masked ones: before near_begin; all
    int kept_all, units;                                   // kept tiles with the last one, which may be short
    __device__ __forceinline__ Work(const SplitArgs& a, int item) : Work(a, item, head_of(a, item / a.row_tiles)) {}
    __device__ __forceinline__ Work(const SplitArgs& a, int item, const Head& head) {
        const AttendCall& c = a.c;
        const int row_tile = item % a.row_tiles, length = head.length;
        t0 = row_tile * kRowTile / c.group;
        t1 = min(c.m - 1, (row_tile * kRowTile + kRowTile - 1) / c.group);
        begin = head.begin;
        kept = head.kept;
        kept_tiles = kept / TA;
        kept_all = kept_tiles + (kept % TA != 0);
        seen = seen_rows(length, c.m, t0, t1, c.window, c.sinks);
        const int hidden = c.window > 0 ? max(0, seen.p1 - c.window + 1 - seen.low) : 0;    // rows from low on that the last token does not see
        first_tiles = seen.first / TB;
        near_tiles = (seen.high - seen.low + TB - 1) / TB;
        near_end = max(0, min(seen.high, seen.p0 + 1) - seen.low) / TB;
        near_begin = min((hidden + TB - 1) / TB, near_end);
        cache_tiles = first_tiles + near_end - near_begin;
        low_masked = (seen.first % TB != 0) + near_begin;
        cache_masked = low_masked + near_tiles - near_end;
        units = max(1, kept_all * kUnitA + (cache_tiles + cache_masked) * kUnitB);   // (nothing to read: still somebody's to write)
    }
    __device__ __forceinline__ int row_of(int tile) const { return tile < first_tiles ? tile * TB : seen.low + (near_begin + tile - first_tiles) * TB; }
};

// Tiles from, from + 4, .. below `end` one after the other, the next one's loads in flight behind the one at hand.
template <int F, class L>
__device__ __forceinline__ void stream(int from, int end, Running& r, const Queries& q, float scale_log2, L load) {
    if (from >= end) return;
    Tile<F> x, y;
    load(x, from, ~0u);
    for (;;) {
        const int next = from + kSplitWaves;
        load(y, next < end ? next : from, next < end ? ~0u : 0u);
        take<F, false>(r, x, q, scale_log2, 0u);
        if (next >= end) return;
        from = next + kSplitWaves;
        load(x, from < end ? from : next, from < end ? ~0u : 0u);
        take<F, false>(r, y, q, scale_log2, 0u);
        if (from >= end) return;
    }
}

__device__ __forceinline__ int ceil_div(int x, int y) { return (x + y - 1) / y; }

// A workgroup's place in the list of all items.
struct Place {
    int item, into, size;              // units of the item in front of the share; of the share (0: nothing to do)
    int end;                           // the share has no part of this item and those after it
    int first, last;                   // workgroups that have a part of the item
    Head head;                         // of the item
};
// Shares of equal size, whatever the heads' lengths: where a share ends inside an item, its neighbour has the rest, and a workgroup may have parts of
// several items.  What it takes to end one item and begin the next, about 4 us, counts as kBetween units in front of an item (windows of 32 sequences with 4 units 82 us, 16
// 75; 8 heads of 4 sequences in 4 bits with 8 units 42, 32 36).  Few items (a.whole): every one
// has workgroups of its own, in proportion to its units, and a share is one part.
// (Every wave for itself: a lane adds up its items, the lanes' sums are added up by shuffles, and the lane that has the share's begin is asked.)
__device__ __forceinline__ int added_up(int x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int y = __shfl_up(x, k);
        if (lane >= k) x += y;
    }
    return x;
}
__device__ __forceinline__ Head head_from(const Head& h, int lane) {
    Head r;
    r.begin = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)h.begin, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(h.begin >> 32), lane) << 32);
    r.kept = __builtin_amdgcn_readlane(h.kept, lane);
    r.length = __builtin_amdgcn_readlane(h.length, lane);
    return r;
}
// Each item its own workgroups: shares of all items that are equal count for more where few share one for long.
__host__ __device__ __forceinline__ bool few_enough(int items, int64_t shares, int64_t tiles) { return 8 * items <= shares || tiles <= 64 * shares; }
template <int FA, int FB>
struct Places {
    static constexpr int kBetween = FA == kMxBf16 || FA == kMxF32 ? 32 : 16, kAtOnce = 4;
    // A lane's items have less than this many units, so that those of 64 lanes do not pass 2^31 (a head's rows count once for each of its row tiles: memory does not bound them).  Where
    // a lane has more, heads are of a million rows at least, or of 140 GB with few items, and every item has one workgroup.
    static constexpr int kMostUnits = (1 << 25) - 2 * kBetween;
    const SplitArgs& a;
    int all, shares, at;               // units of all items; workgroups with a share; units in front of the item at hand, without its kBetween
    bool whole;                        // workgroups have parts of one item each
    __device__ __forceinline__ int begin_of(int share) const { return (int)((int64_t)all * share / shares); }
    __device__ __forceinline__ int share_of(int unit) const { return (int)((((int64_t)unit + 1) * shares - 1) / all); }     // whose share holds a unit
    __device__ __forceinline__ void owners(Place& p, int units) const {
        if (whole) return;
        p.first = share_of(at + kBetween);
        p.last = share_of(at + kBetween + units - 1);
    }
    __device__ __forceinline__ Place find() {
        const int lane = threadIdx.x & 63, each = (a.items + 63) / 64, from = min(lane * each, a.items), end = min(from + each, a.items), block = blockIdx.x;
        Place p{0, 0, 0, a.items, 0, 0, {0, 0, 0}};
        int owner;
        Head head[kAtOnce];
        int units[kAtOnce], mine = 0;
        if (a.whole) {                 // (each == 1)
            head[0] = head_of(a, min(from, a.items - 1) / a.row_tiles);
            mine = lane < a.items ? min(Work<FA, FB>(a, from, head[0]).units, kMostUnits) : 0;
            const int tiles = __builtin_amdgcn_readlane(added_up(mine), 63);
            whole = !__any(mine >= kMostUnits) && few_enough(a.items, a.shares, tiles);
            if (whole) {
                // (the host knows the largest lengths that there may be; here are those that there are: 8 sequences of 250 tokens in caches of 16384 18 us by the caches' size, so 9)
                const int some = min(a.shares, max(a.items, (int)__builtin_sqrtf(a.weight * (float)a.items * (float)tiles)));
                const int parts = lane >= a.items ? 0 : tiles < a.least * 3 / 8 * a.items ? 1 : min(mine, max(1, (int)((int64_t)mine * some / tiles))), parts_up_to = added_up(parts);
                const uint64_t beyond = __ballot(block < parts_up_to);
                if (!beyond) return p;
                owner = __builtin_ctzll(beyond);
                const int n = __builtin_amdgcn_readlane(parts, owner), units = __builtin_amdgcn_readlane(mine, owner);
                p.first = __builtin_amdgcn_readlane(parts_up_to, owner) - n;
                p.last = p.first + n - 1;
                p.into = (int)((int64_t)units * (block - p.first) / n);
                p.size = (int)((int64_t)units * (block - p.first + 1) / n) - p.into;
                p.item = owner;
                p.head = head_from(head[0], owner);
                return p;
            }
            if (lane < a.items) mine += kBetween;
            units[0] = mine;
#pragma unroll
            for (int k = 1; k < kAtOnce; ++k) units[k] = 0, head[k] = head[0];
        }
        // (the loads of four items at a time)
        for (int i = a.whole ? end : from; i < end; i += kAtOnce) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) head[k] = head_of(a, min(i + k, a.items - 1) / a.row_tiles);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                units[k] = i + k < end ? Work<FA, FB>(a, i + k, head[k]).units + kBetween : 0;
                mine = min(mine + units[k], kMostUnits);
            }
        }
        const int up_to = added_up(mine);
        all = __builtin_amdgcn_readlane(up_to, 63);
        const int tiles = all - a.items * kBetween;
        if (tiles < a.least * a.items || __any(mine >= kMostUnits)) {  // little to read, in fact, or more than is counted: items as they are
            const int places = min(a.items, a.shares);
            p.item = (int)((int64_t)a.items * block / places);
            p.end = (int)((int64_t)a.items * (block + 1) / places);
            if (block < places) p.head = head_of(a, p.item / a.row_tiles), p.size = INT_MAX;
            return p;
        }
        // (no more shares than tiles: none may be without any between two that have parts of one item)
        shares = max(1, min(a.shares, (all - a.items * kBetween) / (kBetween + 1)));
        const int begin = begin_of(block);
        if (block >= shares) return p;
        p.size = begin_of(block + 1) - begin;
        owner = __builtin_ctzll(__ballot(begin < up_to));
        int front = up_to - mine, i = from;
        if (each <= kAtOnce) {         // (in its lane's registers)
            Head mine_head = head[0];
#pragma unroll
            for (int k = 0; k + 1 < kAtOnce; ++k)
                if (i == from + k && begin >= front + units[k]) {
                    front += units[k];
                    ++i;
                    mine_head = head[k + 1];
                }
            p.item = __builtin_amdgcn_readlane(i, owner);
            at = __builtin_amdgcn_readlane(front, owner);
            p.head = head_from(mine_head, owner);
        } else {
            p.item = owner * each;
            at = __builtin_amdgcn_readlane(front, owner);
            for (;; ++p.item) {
                p.head = head_of(a, p.item / a.row_tiles);
                const int n = Work<FA, FB>(a, p.item, p.head).units + kBetween;
                if (begin < at + n) break;
                at += n;
            }
        }
        p.into = begin - at - kBetween;
        if (p.into < 0) {              // the share begins in front of the item
            p.size += p.into;
            p.into = 0;
        }
        return p;
    }
};

__device__ __forceinline__ void store_shared(uint64_t* to, f32x2a x) {
    __hip_atomic_store(to, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2a load_shared(const uint64_t* from) {
    return __builtin_bit_cast(f32x2a, __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Eight channels of row R's result, o un-normalised.
template <int FB>
__device__ __forceinline__ void write_row(const AttendCall& c, int g, int R, int d0, float* o, float top, float sum) {
    const bool empty = sum == 0.f;
    const float over = empty ? 0.f : 1.f / sum;
    const int b = g / c.kv, t = R / c.group, h = (g - b * c.kv) * c.group + R % c.group;
    const int64_t out_row = ((int64_t)b * c.m + t) * c.kv * c.group + h;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= over;
    if (FB == kBf16) {
        *(u32x4a*)((char*)c.out + out_row * 256 + d0 * 2) = (u32x4a){pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7])};
    } else {
        *(f32x4a*)((char*)c.out + out_row * 512 + d0 * 4) = (f32x4a){o[0], o[1], o[2], o[3]};
        *(f32x4a*)((char*)c.out + out_row * 512 + d0 * 4 + 16) = (f32x4a){o[4], o[5], o[6], o[7]};
    }
    if (c.lse && d0 == 0) c.lse[((int64_t)b * c.kv * c.group + h) * c.m + t] = empty ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// The four waves' parts in LDS of the rows that 16 threads of 8 channels each take, put together.
typedef float WaveParts[kSplitWaves][kRowTile][128 + 4];
typedef float WaveValues[kSplitWaves][kRowTile];
__device__ __forceinline__ void merge_waves(const WaveParts& part, const WaveValues& tops, const WaveValues& sums, int row, int d0, float* o, float& top, float& sum) {
    top = tops[0][row];
#pragma unroll
    for (int w = 1; w < kSplitWaves; ++w) top = fmaxf(top, tops[w][row]);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) {
        const float weight = __builtin_amdgcn_exp2f(tops[w][row] - top);
        sum += weight * sums[w][row];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] += weight * part[w][row][d0 + i];
    }
}

// Joins workgroups w0 .. w1's parts of an item: 16 lanes a row; the 16 threads' groups of a workgroup share out the parts where there are fewer rows.
template <int FB>
__device__ __forceinline__ void join(const SplitArgs& a, int item, int w0, int w1, WaveParts& part, WaveValues& tops, WaveValues& sums) {
    const int g = item / a.row_tiles, R0 = (item - g * a.row_tiles) * kRowTile, rows = min(kRowTile, a.rows - R0), group = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 8;
    const int ways = rows <= 4 ? 4 : rows <= 8 ? 2 : 1, row = group % (kRowTile / ways), way = group / (kRowTile / ways);
    float top = kNoScore, sum = 0.f, o[8] = {};
    if (row < rows)
        for (int first = w0 + way; first <= w1; first += 8 * ways) {
            // (eight parts' loads together; the last one again for those beyond it, left out)
            f32x2a ml[8], x[8][4];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t at = ((int64_t)min(first + k * ways, w1) + item) * kRowTile + row;
                ml[k] = load_shared((const uint64_t*)(a.part_ml + at));
#pragma unroll
                for (int i = 0; i < 4; ++i) x[k][i] = load_shared((const uint64_t*)(a.part_o + at * 128 + d0) + i);
            }
            float next = top;
#pragma unroll
            for (int k = 0; k < 8; ++k) next = fmaxf(next, ml[k].x);
            const float keep = __builtin_amdgcn_exp2f(top - next);
            sum *= keep;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] *= keep;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (first + k * ways > w1) continue;
                const float weight = __builtin_amdgcn_exp2f(ml[k].x - next);
                sum += weight * ml[k].y;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] += weight * x[k][i / 2][i % 2];
            }
            top = next;
        }
    if (ways > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) part[way][row][d0 + i] = o[i];
        if (d0 == 0) tops[way][row] = top, sums[way][row] = sum;
        __syncthreads();
        if (way > 0 || row >= rows) return;
        for (int w = 1; w < ways; ++w) {
            const float other = tops[w][row], next = fmaxf(top, other);
            const float keep = __builtin_amdgcn_exp2f(top - next), weight = __builtin_amdgcn_exp2f(other - next);
            sum = sum * keep + weight * sums[w][row];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = o[i] * keep + weight * part[w][row][d0 + i];
            top = next;
        }
    }
    if (row < rows && way == 0) write_row<FB>(a.c, g, R0 + row, d0, o, top, sum);
}

// An item that the workgroup has a part of, and the workgroups that have others.
struct Part {
    int item, first, last;
};

template <int FA, int FB, bool PAST>
__global__ __launch_bounds__(kSplitWaves * 64, 2) void attend_split_kernel(SplitArgs a) {
    __shared__ __attribute__((aligned(16))) WaveParts part;
    __shared__ WaveValues tops, sums;
    __shared__ bool last[2];
    Part begun{-1, 0, 0}, ended{-1, 0, 0};                  // items that another workgroup has begun, or ends
    const AttendCall& c = a.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    constexpr int kBytes = FB == kBf16 ? 2 : 4;
    Places<FA, FB> places{a, 0, 0, 0, false};
    Place place{(int)blockIdx.x, 0, 0, a.items, 0, 0, {0, 0, 0}};
    if (a.shares > 0) {
        place = places.find();
        if (place.size <= 0) return;
    } else {
        place.head = head_of(a, place.item / a.row_tiles);
    }
    for (int item = place.item;; ++item) {
        const Work<FA, FB> work(a, item, place.head);
        const int lo = a.shares > 0 ? place.into : 0, hi = a.shares > 0 ? lo + min(work.units - lo, place.size) : work.units;
        const int g = item / a.row_tiles, row_tile = item - g * a.row_tiles, b = g / c.kv, head = g % c.kv;

        // this lane's query row (rows beyond the last repeat it; nothing of them is written)
        const int R = min(row_tile * kRowTile + col, a.rows - 1), t = R / c.group;
        const char* q_row = (const char*)c.Q + ((((int64_t)b * c.m + t) * c.kv + head) * c.group + R % c.group) * (128 * kBytes);
        Queries q;
        Running r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.o[i] = (f32x4a){0, 0, 0, 0};
        r.top = kNoScore;
        r.sum = 0.f;

        if constexpr (FA != kNone) {
            constexpr int T = Tile<FA>::T;
            const int from = min(ceil_div(lo, work.kUnitA), work.kept_all), end = min(ceil_div(hi, work.kUnitA), work.kept_all);
            if (from < end) {
                Tile<FA>::queries(q, q_row, quarter);
                stream<FA>(from + wave, min(end, work.kept_tiles), r, q, a.scale_log2, [&](Tile<FA>& x, int tile, uint32_t on) {
                    x.template load<PAST>(c.K_kept, c.V_kept, c.K_scales, c.V_scales, work.begin + (int64_t)tile * T, T, lane, on);
                });
                if (end > work.kept_tiles && wave == (work.kept_tiles - from) % kSplitWaves) {
                    const int left = work.kept - work.kept_tiles * T;
                    Tile<FA> x;
                    x.template load<PAST>(c.K_kept, c.V_kept, c.K_scales, c.V_scales, work.begin + (int64_t)work.kept_tiles * T, left, lane);
                    take<FA, true>(r, x, q, a.scale_log2, (1u << min(max(left - quarter * (T / 4), 0), T / 4)) - 1u);
                }
            }
        }
        constexpr int T = Tile<FB>::T;
        const int all = work.cache_tiles + work.cache_masked, before = work.kept_all * work.kUnitA;
        const int from = min(ceil_div(max(lo - before, 0), work.kUnitB), all), end = min(ceil_div(max(hi - before, 0), work.kUnitB), all);
        if (from < end) {
            const int64_t base = (int64_t)g * c.stride;
            Tile<FB>::queries(q, q_row, quarter);
            stream<FB>(from + wave, min(end, work.cache_tiles), r, q, a.scale_log2,
                       [&](Tile<FB>& x, int tile, uint32_t on) { x.template load<PAST>(c.K, c.V, nullptr, nullptr, base + work.row_of(tile), T, lane, on); });
            const int masked = max(from, work.cache_tiles) - work.cache_tiles, turn = (max(from, work.cache_tiles) - from) % kSplitWaves;
            for (int i = masked + (wave - turn + kSplitWaves) % kSplitWaves; i < end - work.cache_tiles; i += kSplitWaves) {
                const int near = i < work.low_masked ? i - (work.seen.first % T != 0) : work.near_end + i - work.low_masked;        // -1: the end of the first rows
                const int j0 = near < 0 ? work.first_tiles * T : work.seen.low + near * T, count = min(T, (near < 0 ? work.seen.first : work.seen.high) - j0);
                const int p = work.seen.p0 + (t - work.t0);
                Tile<FB> x;
                x.template load<PAST>(c.K, c.V, nullptr, nullptr, base + j0, count, lane);
                uint32_t mask = 0;
#pragma unroll
                for (int e = 0; e < T / 4; ++e) {
                    const int k = quarter * (T / 4) + e;
                    mask |= k < count && sees(p, j0 + k, c.window, c.sinks) ? 1u << e : 0u;
                }
                take<FB, true>(r, x, q, a.scale_log2, mask);
            }
        }

        // the four waves' parts
        r.sum = quarters_sum(r.sum);
        if (quarter == 0) {
            tops[wave][col] = r.top;
            sums[wave][col] = r.sum;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float* to = &part[wave][col][eight_of(quarter * 4 + j) * 8];
            *(f32x4a*)to = (f32x4a){r.o[0][j], r.o[1][j], r.o[2][j], r.o[3][j]};
            *(f32x4a*)(to + 4) = (f32x4a){r.o[4][j], r.o[5][j], r.o[6][j], r.o[7][j]};
        }
        __syncthreads();
        const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 8;
        const int Rw = row_tile * kRowTile + row;
        if (Rw < a.rows) {
            float o[8], top, sum;
            merge_waves(part, tops, sums, row, d0, o, top, sum);
            if (lo > 0 || hi < work.units) {
                // (past the caches of this XCD: atomic stores and loads of the device's scope are coherent between them)
                const int64_t at = ((int64_t)blockIdx.x + item) * kRowTile + row;
                uint64_t* to = (uint64_t*)(a.part_o + at * 128 + d0);
#pragma unroll
                for (int i = 0; i < 4; ++i) store_shared(to + i, f32x2a{o[2 * i], o[2 * i + 1]});
                if (d0 == 0) store_shared((uint64_t*)(a.part_ml + at), f32x2a{top, sum});
            } else {
                write_row<FB>(c, g, Rw, d0, o, top, sum);
            }
        }
        if (a.shares == 0) return;
        if (lo > 0 || hi < work.units) {                   // (the first or the last of this workgroup's items)
            places.owners(place, work.units);
            (lo > 0 ? begun : ended) = Part{item, place.first, place.last};
        }
        places.at += work.units + places.kBetween;
        place.size -= hi - lo + places.kBetween;
        place.into = 0;
        if (place.size <= 0 || item + 1 >= place.end) break;
        place.head = head_of(a, (item + 1) / a.row_tiles);
        __syncthreads();                                   // (part, tops and sums are read)
    }
    // Of all workgroups that have a part of an item, the last one to be done joins them.  Its parts must have arrived before it is counted, and a barrier alone
    // does not wait for stores to memory: every wave waits for its own.  They went past the caches, and are read past them, so nothing is left to be
    // written back or dropped (with fences of the device's scope, which do both: 20 sequences of 4 bits 105 -> 145 us, one token 17 -> 27).
    dma_wait();
    __syncthreads();
    if (threadIdx.x == 0) {
        last[0] = begun.item >= 0 && __hip_atomic_fetch_add(&a.arrived[begun.item], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == begun.last - begun.first;
        last[1] = ended.item >= 0 && __hip_atomic_fetch_add(&a.arrived[ended.item], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == ended.last - ended.first;
    }
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < 2; ++k)
        if (last[k]) {
            const Part& p = k == 0 ? begun : ended;
            join<FB>(a, p.item, p.first, p.last, part, tops, sums);
            if (threadIdx.x == 0) __hip_atomic_store(&a.arrived[p.item], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
        }
}

template <int FA, int FB, bool PAST>
hipError_t launch(const SplitArgs& a, hipStream_t stream) {
    attend_split_kernel<FA, FB, PAST><<<(unsigned)(a.whole ? a.shares + a.items : a.shares > 0 ? a.shares : a.items), kSplitWaves * 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_split(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream) {
    SplitArgs a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.rows = call.m * call.group;
    a.row_tiles = (a.rows + kRowTile - 1) / kRowTile;
    a.items = (int)(call.count * call.kv * a.row_tiles);
    // How many workgroups share the tiles (as far as the host knows them) of all items; 0: every item has one.
    const bool mx = call.K_scales != nullptr, f32 = call.dtype == CURDKV_DTYPE_F32;
    const int T = mx && !f32 ? 32 : 16, row = f32 ? 512 : 256;
    const int64_t units = ctx->num_cu, heads = call.count * call.kv, slot = kRowTile * kPartBytes;
    const int64_t keys = call.window > 0 ? std::min((int64_t)call.n, (int64_t)call.window + call.sinks + call.m) : call.n;
    const int64_t tiles = (call.rows / T + heads * (keys / T + 1)) * a.row_tiles, room = call.scratch ? (call.scratch_bytes - kScratchCounters) / slot : 0;
    // One a unit at most (two: one token over 131072 rows 100 us, so 91).  4 bits, whose expansion wants two waves a SIMD, two a unit
    // where they have long to go (320 us, so 295; 32 tiles a unit: 18, 20).  A tile a wave at least, and no more parts of an item than pay: its tiles over the parts are read
    // in a time of their own, its parts are counted and joined in theirs, and the two together are least where parts^2 is about the tiles, or twice them in fp32 (one token of 8
    // heads over 4000 rows 14.7 us with as many as there are units, so 13.1; in 4 bits 18.2, so 13.1; of one head over 16000 48.5, so 17.1).
    a.weight = f32 ? 2.f : 1.f;
    const int64_t most = (int64_t)std::sqrt((double)a.weight * a.items * tiles);
    const int64_t wanted = std::min(units * (mx && tiles >= 1024 * units ? 2 : 1), std::max((int64_t)a.items, std::min(most, (tiles + kSplitWaves - 1) / kSplitWaves)));
    // (slots of partial results: a workgroup and an item add up to less than shares + items, and than shares + 2 items where every item has workgroups of its own, of which
    // there may be shares + items)
    const int64_t between = (a.items <= 64 ? 2 : 1) * (int64_t)a.items;
    int64_t shares = std::min(wanted, room - between);
    // Few items: each its own workgroups, which have less to look up and to join (64 heads of up to 2000 rows 18.1 us, so 15.6, of 4 bits 21.5, so 14.7); where few share one
    // for long, equal shares of all of them count for more (64 heads of 16000 in 4 bits 41, so 49).
    a.whole = a.items <= 64 && 2 * a.items <= shares;
    // To share costs a join: 3 us, 10 where a workgroup may have parts of several items.  Not shared and shared, us: 8 heads of 500 rows 8.6 and 10.1, of
    // 1000 12.9 and 11.2; 64 of up to 500 8.8 and 11.1, of 1000 13.3 and 12.7; 256 of 500 10 and 20, of 2000 32 and 36, of 8000 102 and 91; 1024 of 1000 57 and
    // 65, of 2000 109 and 100.  fp32's tiles take twice as long: 8 of 250 11.6 and 12.3, of 400 14.9 and 13.2; 128 of 1000 28 and 27.  Kept rows differ more from head to
    // head: 8 of about 250 11.3 and 10.9, 400 in 4 bits 10.5 and 11.1, 600 12.8 and 11.0; 256 of 500 27.9 and 26.4, of 1000 61 and 40, in 4 bits 26.6 and 24.3.
    a.least = 128 / (f32 ? 2 : 1) / (call.offsets ? 4 : 1);
    // More items than find() holds in registers, four a lane, are looked up one after the other: 10 us and more.  Uneven kept rows, not shared and shared: in 4 bits 384 heads of
    // 1000 25 and 33, of 1500 35 and 31, 1536 of 1000 56 and 89, of 2000 107 and 104, 3200 of 1000 101 and 143, of 3000 248 and 234; in bf16 1536 of 500 91 and 106, of 1000 169 and 139,
    // 3200 of 1000 340 and 271; 3200 of 300 in 4 bits under fp32 132 and 176.
    if (call.offsets && a.items > 4 * 64) a.least += (mx && !f32 ? 16 : 0) + (a.items - 256) / 128;
    const int64_t least = a.whole && few_enough(a.items, shares, tiles) ? a.least * 3 / 8 : a.least;
    // Equal ones in whole turns of all units are shared out already: 256 heads of 4000 rows 81 and 87, through windows of 4096 69 and 74 (264 heads: 106 and 77).
    const bool equal = !call.offsets && (!call.lengths || (call.window > 0 && 2 * (int64_t)call.window <= call.n)) && a.items % units == 0;
    if (tiles < least * a.items || equal || a.items > kCounters || (shares < wanted && shares < a.items)) shares = 0;
    a.shares = (int)shares;
    a.whole = a.whole && shares > 0;
    a.arrived = (int*)call.scratch;
    a.part_o = (float*)(a.arrived + kCounters);
    a.part_ml = (f32x2a*)(a.part_o + (shares + between) * kRowTile * 128);
    // (bytes that 256 MB of Infinity Cache would not hold until the next call: one token over 131072 rows 105 us through the caches, 91 past them; 64 tokens in fp32 over 4000
    // rows, which 16 tiles of their rows read one after the other, 59 and 75)
    const bool past = 2 * ((mx ? 68 : row) * call.rows + row * heads * keys) > kPastCaches;
    if (mx) {
        if (past) return f32 ? launch<kMxF32, kF32, true>(a, stream) : launch<kMxBf16, kBf16, true>(a, stream);
        return f32 ? launch<kMxF32, kF32, false>(a, stream) : launch<kMxBf16, kBf16, false>(a, stream);
    }
    if (!call.offsets) {
        if (past) return f32 ? launch<kNone, kF32, true>(a, stream) : launch<kNone, kBf16, true>(a, stream);
        return f32 ? launch<kNone, kF32, false>(a, stream) : launch<kNone, kBf16, false>(a, stream);
    }
    if (past) return f32 ? launch<kF32, kF32, true>(a, stream) : launch<kBf16, kBf16, true>(a, stream);
    return f32 ? launch<kF32, kF32, false>(a, stream) : launch<kBf16, kBf16, false>(a, stream);
}

}  // namespace curdkv
