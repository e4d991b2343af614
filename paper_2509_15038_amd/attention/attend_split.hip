// Attention of a few tokens over long caches: the rows of a KV head are shared out over workgroups, whose results a second
// kernel joins.  out = softmax(q k / sqrt(d)) v with the running maximum M and sum L of a softmax: of two parts of the keys
// with (M1, L1, o1) and (M2, L2, o2), o un-normalised, the whole has M = max, L = L1 2^(M1-M) + L2 2^(M2-M) and o likewise
// (scores in units of log 2 throughout).
//
// HBM-bound: every cache row is read once, by one wave, straight into the operand registers; nothing of the cache passes LDS.
// S^T = K Q^T: the rows of 16 keys are the A operand of mfma_f32_16x16x32_bf16 (16x16x4 for fp32), the 16 rows R of the queries
// the B operand, so that a lane holds scores of one R for the keys of its quarter of the wave.  Which key a row of the A operand
// stands for is free: they are picked so that a lane's scores are of T/4 consecutive keys, exactly what the B operand of
// O^T = V^T P^T wants of its lane, and P never leaves its registers.  V rows are loaded whole, 16 lanes of 8 channels a row,
// a lane holding the same 8 channels of the T/4 keys of its quarter; v_perm pairs them up into the A operand of eight products,
// product i for channels 8 c + i.

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

constexpr int kSplitWaves = 4;
constexpr int kRowTile = 16;           // rows R a workgroup handles
constexpr int64_t kPartBytes = 128 * sizeof(float) + 2 * sizeof(float);     // of a row of partial results
constexpr int64_t kPartRows = CURDKV_ATTEND_SCRATCH_BYTES / kPartBytes;

struct SplitArgs {
    AttendCall c;
    float scale_log2;
    int groups, rows, row_tiles;       // count * kv; m * group; tiles of them
    int shares, chunk;                 // workgroups a head and row tile; tiles of keys in a row
    float* part_o;                     // [groups * rows][shares][128]
    f32x2a* part_ml;                   // [groups * rows][shares]: maximum, sum
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
__device__ __forceinline__ float unit_of(uint32_t scale) { return __uint_as_float(scale << 23); }   // (2^-127 comes out as 0: it stands for zeros)

// A lane's part of the running softmax: column R = lane % 16, channels 32 (lane / 16) + 8 j + i in o[i][j].
struct Running {
    f32x4a o[8];
    float top, sum;                    // of R so far (top: of all quarters; sum: of the lane's keys)
};

// o += V^T P^T for bf16 rows: v[e] the lane's 8 channels of key e of its quarter, p[e] that key's weights.
__device__ __forceinline__ f32x4a product(u32x4a x, u32x4a y, f32x4a z) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8a, x), __builtin_bit_cast(bf16x8a, y), z, 0, 0, 0);
}
__device__ __forceinline__ void add_values(const u32x4a* v, const float* p, f32x4a* o) {
    u32x4a pb;
#pragma unroll
    for (int u = 0; u < 4; ++u) pb[u] = pack_bf16(p[2 * u], p[2 * u + 1]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        u32x4a even, odd;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            even[u] = __builtin_amdgcn_perm(v[2 * u + 1][w], v[2 * u][w], 0x05040100u);
            odd[u] = __builtin_amdgcn_perm(v[2 * u + 1][w], v[2 * u][w], 0x07060302u);
        }
        o[2 * w] = product(even, pb, o[2 * w]);
        o[2 * w + 1] = product(odd, pb, o[2 * w + 1]);
    }
}
// (fp32 products: exact to 2^-24 a product, 1/16 of the bf16 rate, which the rows' bytes still hide)
__device__ __forceinline__ void add_values(const float (*v)[8], const float* p, f32x4a* o) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][i], p[e], o[i], 0, 0, 0);
}

// Infinities and NaN in rows that some R does not see must not meet its zero weight.  Zeros take their place, and the R that do see one
// (seen: a bit for each of the lane's keys) get it whatever its weight: where a product of "is such a value" with "is seen" is not zero.
constexpr uint32_t kInf16 = 0x7F80u;
__device__ __forceinline__ bool any_not_finite(const u32x4a* v) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) bad |= (v[e][w] & kInf16) == kInf16 || (v[e][w] & (kInf16 << 16)) == kInf16 << 16;
    return __any(bad);
}
__device__ __forceinline__ bool any_not_finite(const float (*v)[8]) {
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
__device__ __forceinline__ void spread_not_finite(u32x4a* v, uint32_t seen, f32x4a* o) {
    u32x4a sees;
#pragma unroll
    for (int u = 0; u < 4; ++u) sees[u] = (seen >> (2 * u) & 1 ? 0x3F80u : 0u) | (seen >> (2 * u + 1) & 1 ? 0x3F800000u : 0u);
#pragma unroll 1
    for (uint32_t kind = 0; kind < 3; ++kind) {
        const float value = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4a has;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t x = v[2 * u][w] >> (16 * h) & 0xFFFFu, y = v[2 * u + 1][w] >> (16 * h) & 0xFFFFu;
                    has[u] = (kind_of(x, kInf16, 0x8000u) == kind ? 0x3F80u : 0u) | (kind_of(y, kInf16, 0x8000u) == kind ? 0x3F800000u : 0u);
                }
                const f32x4a z = product(has, sees, (f32x4a){0, 0, 0, 0});
#pragma unroll
                for (int j = 0; j < 4; ++j) o[2 * w + h][j] += z[j] > 0.f ? value : 0.f;
            }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if ((v[e][w] & kInf16) == kInf16) v[e][w] &= 0xFFFF0000u;
            if ((v[e][w] & (kInf16 << 16)) == kInf16 << 16) v[e][w] &= 0xFFFFu;
        }
}
__device__ __forceinline__ void spread_not_finite(float (*v)[8], uint32_t seen, f32x4a* o) {
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
__device__ __forceinline__ void add_values_masked(V* v, const float* p, uint32_t seen, f32x4a* o) {
    if (any_not_finite(v)) spread_not_finite(v, seen, o);
    add_values(v, p, o);
}

// One tile of T keys in registers.  `first`: row of its first key in K and V; `count`: keys of it that there are (>= 1), the last
// one stands in for those beyond.  MASKED: some key of it is hidden from some R.
template <int F> struct Tile;

template <>
struct Tile<kBf16> {
    static constexpr int T = 32;
    u32x4a k[2][4], v[8];
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t*, const uint8_t*, int64_t first, int count, int lane) {
        const int c = lane & 15, quarter = lane >> 4;
        const char* Kb = (const char*)K + first * 256;
        const char* Vb = (const char*)V + first * 256;
        if (count == T) {
            const uint32_t k_at = (c >> 2) * 2048 + (c & 3) * 256 + quarter * 16, v_at = quarter * 2048 + c * 16;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < 4; ++s) k[t][s] = *(const u32x4a*)(Kb + k_at + t * 1024 + s * 64);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = *(const u32x4a*)(Vb + v_at + e * 256);
            return;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = min((c >> 2) * 8 + t * 4 + (c & 3), count - 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) k[t][s] = *(const u32x4a*)(Kb + (uint32_t)(key * 256 + (s * 4 + quarter) * 16));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = *(const u32x4a*)(Vb + (uint32_t)(min(quarter * 8 + e, count - 1) * 256 + c * 16));
    }
    __device__ __forceinline__ static void queries(Queries& q, const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 4; ++s) q.q[s] = ((const u32x4a*)row)[s * 4 + quarter];
    }
    __device__ __forceinline__ void scores(const Queries& q, float* s) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4a a = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) a = product(k[t][i], q.q[i], a);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[t * 4 + j] = a[j];
        }
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
    f32x4a k[8];
    float v[4][8];
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t*, const uint8_t*, int64_t first, int count, int lane) {
        const int c = lane & 15, quarter = lane >> 4;
        const char* Kb = (const char*)K + first * 512;
        const char* Vb = (const char*)V + first * 512;
        const uint32_t k_at = min(c, count - 1) * 512 + quarter * 16;
#pragma unroll
        for (int s = 0; s < 8; ++s) k[s] = *(const f32x4a*)(Kb + k_at + s * 64);
        if (count == T) {
            const uint32_t v_at = quarter * 2048 + c * 32;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                *(f32x4a*)&v[e][0] = *(const f32x4a*)(Vb + v_at + e * 512);
                *(f32x4a*)&v[e][4] = *(const f32x4a*)(Vb + v_at + e * 512 + 16);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const char* row = Vb + (uint32_t)(min(quarter * 4 + e, count - 1) * 512 + c * 32);
            *(f32x4a*)&v[e][0] = *(const f32x4a*)row;
            *(f32x4a*)&v[e][4] = *(const f32x4a*)(row + 16);
        }
    }
    __device__ __forceinline__ static void queries(Queries& q, const void* row, int quarter) {
#pragma unroll
        for (int s = 0; s < 8; ++s) q.q[s] = ((const u32x4a*)row)[s * 4 + quarter];
    }
    __device__ __forceinline__ void scores(const Queries& q, float* s) const {
        f32x4a a = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][j], __uint_as_float(q.q[i][j]), a, 0, 0, 0);
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
    u32x4a k[2];
    uint32_t v[8];
    uint32_t ks[2], vs[8];
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t* Ks, const uint8_t* Vs, int64_t first, int count, int lane) {
        const int c = lane & 15, quarter = lane >> 4;
        const char* Kb = (const char*)K + first * 64;
        const char* Vb = (const char*)V + first * 64;
        const uint8_t* Kc = Ks + first * 4;
        const uint8_t* Vc = Vs + first * 4;
        if (count == T) {
            const uint32_t key = (c >> 2) * 8 + (c & 3), k_at = key * 64 + quarter * 16, v_at = quarter * 512 + c * 4;
            const uint32_t ks_at = key * 4 + quarter, vs_at = quarter * 32 + (c >> 2);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                k[t] = *(const u32x4a*)(Kb + k_at + t * 256);
                ks[t] = *(Kc + ks_at + t * 16);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = *(const uint32_t*)(Vb + v_at + e * 64);
                vs[e] = *(Vc + vs_at + e * 4);
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
            const int key = min(quarter * 8 + e, count - 1);
            v[e] = *(const uint32_t*)(Vb + (uint32_t)(key * 64 + c * 4));
            vs[e] = Vc[(uint32_t)(key * 4 + (c >> 2))];
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
        u32x4a x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float unit = unit_of(vs[e]);
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
    __device__ __forceinline__ void load(const void* K, const void* V, const uint8_t* Ks, const uint8_t* Vs, int64_t first, int count, int lane) {
        const int c = lane & 15, quarter = lane >> 4;
        const int key = min(c, count - 1);
        k = *(const u32x4a*)((const char*)K + first * 64 + (uint32_t)(key * 64 + quarter * 16));
        ks = (Ks + first * 4)[(uint32_t)(key * 4 + quarter)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = min(quarter * 4 + e, count - 1);
            v[e] = *(const uint32_t*)((const char*)V + first * 64 + (uint32_t)(row * 64 + c * 4));
            vs[e] = (Vs + first * 4)[(uint32_t)(row * 4 + (c >> 2))];
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
        const float keep = top > r.top ? __builtin_amdgcn_exp2f(r.top - top) : 1.f;       // (-inf before the first key: 0)
        r.sum *= keep;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.o[i] *= keep;
        r.top = top;
    }
    const float off = MASKED && r.top == -INFINITY ? 0.f : r.top;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale_log2, -off));
        r.sum += s[e];
    }
    x.template values<MASKED>(s, seen, r.o);
}

// What a (head, row tile) has to read: tiles that all its R see all of, in chunks, from the kept rows, the first rows and the rows near; and
// tiles to be masked: the ends of those three, and where the window's edge and the diagonal pass.
template <int FA, int FB>
struct Work {
    static constexpr int TA = Tile<FA == kNone ? kBf16 : FA>::T, TB = Tile<FB>::T;
    int64_t begin = 0, kept = 0, kept_tiles = 0, kept_chunks = 0;
    Seen seen;
    int t0, t1;
    int first_tiles, near_begin, near_end, near_tiles;     // whole first rows; of the tiles from seen.low on: whole ones, and all
    int cache_tiles, cache_chunks;                         // whole ones of the cache
    int low_masked, cache_masked;                          // masked ones: before near_begin; all
    __device__ __forceinline__ Work(const SplitArgs& a, int g, int row_tile) {
        const AttendCall& c = a.c;
        t0 = row_tile * kRowTile / c.group;
        t1 = min(c.m - 1, (row_tile * kRowTile + kRowTile - 1) / c.group);
        if (FA != kNone) {
            begin = min(max(c.offsets[g], (int64_t)0), c.total);
            kept = min(max(c.offsets[g + 1], begin), c.total) - begin;
            kept_tiles = kept / TA;
            kept_chunks = (kept_tiles + a.chunk - 1) / a.chunk;
        }
        const int length = c.n > 0 ? (c.lengths ? min(max(c.lengths[g / c.kv], 0), c.n) : c.n) : 0;
        seen = seen_rows(length, c.m, t0, t1, c.window, c.sinks);
        const int hidden = c.window > 0 ? max(0, seen.p1 - c.window + 1 - seen.low) : 0;    // rows from low on that the last token does not see
        first_tiles = seen.first / TB;
        near_tiles = (seen.high - seen.low + TB - 1) / TB;
        near_end = max(0, min(seen.high, seen.p0 + 1) - seen.low) / TB;
        near_begin = min((hidden + TB - 1) / TB, near_end);
        cache_tiles = first_tiles + near_end - near_begin;
        cache_chunks = (cache_tiles + a.chunk - 1) / a.chunk;
        low_masked = (seen.first % TB != 0) + near_begin;
        cache_masked = low_masked + near_tiles - near_end;
    }
    __device__ __forceinline__ int shares(const SplitArgs& a) const { return (int)min((int64_t)a.shares, max((int64_t)1, kept_chunks + cache_chunks)); }
    __device__ __forceinline__ int row_of(int tile) const { return tile < first_tiles ? tile * TB : seen.low + (near_begin + tile - first_tiles) * TB; }
};

// Which whole tiles a wave takes: chunks first, first + shares, ..; of each its tiles wave, wave + 4, ..
struct Walk {
    int64_t chunk, chunks, tiles;
    int shares, per, at, wave;
    __device__ __forceinline__ Walk(int64_t first, int64_t chunks_, int64_t tiles_, int shares_, int chunk_tiles, int wave_)
        : chunk(first), chunks(chunks_), tiles(tiles_), shares(shares_), per(chunk_tiles), at(wave_), wave(wave_) {}
    __device__ __forceinline__ int64_t next() {            // -1: no more
        for (;;) {
            if (chunk >= chunks) return -1;
            const int64_t tile = chunk * per + at;
            if (at < per && tile < tiles) {
                at += kSplitWaves;
                return tile;
            }
            at = wave;
            chunk += shares;
        }
    }
};

// The walk's tiles one after the other, the next one's loads in flight behind the one at hand.
template <int F, class L>
__device__ __forceinline__ void stream(Walk walk, Running& r, const Queries& q, float scale_log2, L load) {
    Tile<F> x, y;
    int64_t tx = walk.next(), ty;
    if (tx < 0) return;
    load(x, tx);
    for (;;) {
        ty = walk.next();
        load(y, ty < 0 ? tx : ty);
        take<F, false>(r, x, q, scale_log2, 0u);
        if (ty < 0) return;
        tx = walk.next();
        load(x, tx < 0 ? ty : tx);
        take<F, false>(r, y, q, scale_log2, 0u);
        if (tx < 0) return;
    }
}

template <int FA, int FB>
__global__ __launch_bounds__(kSplitWaves * 64, 2) void attend_split_kernel(SplitArgs a) {
    __shared__ __attribute__((aligned(16))) float part[kSplitWaves][kRowTile][128 + 4];
    __shared__ float tops[kSplitWaves][kRowTile], sums[kSplitWaves][kRowTile];
    const AttendCall& c = a.c;
    const int share = blockIdx.x % a.shares;
    const int g = blockIdx.x / a.shares % a.groups, row_tile = blockIdx.x / a.shares / a.groups;
    const Work<FA, FB> work(a, g, row_tile);
    const int shares = work.shares(a);
    if (share >= shares) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    const int b = g / c.kv, head = g % c.kv;
    constexpr int kBytes = FB == kBf16 ? 2 : 4;

    // this lane's query row (rows beyond the last repeat it; nothing of them is written)
    const int R = min(row_tile * kRowTile + col, a.rows - 1), t = R / c.group;
    const char* q_row = (const char*)c.Q + ((((int64_t)b * c.m + t) * c.kv + head) * c.group + R % c.group) * (128 * kBytes);
    Queries q;
    Running r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.o[i] = (f32x4a){0, 0, 0, 0};
    r.top = -INFINITY;
    r.sum = 0.f;

    if constexpr (FA != kNone) {
        constexpr int T = Tile<FA>::T;
        Tile<FA>::queries(q, q_row, quarter);
        stream<FA>(Walk(share, work.kept_chunks, work.kept_tiles, shares, a.chunk, wave), r, q, a.scale_log2, [&](Tile<FA>& x, int64_t tile) {
            x.load(c.K_kept, c.V_kept, c.K_scales, c.V_scales, work.begin + tile * T, T, lane);
        });
        const int left = (int)(work.kept - work.kept_tiles * T);
        if (left > 0 && share == shares - 1 && wave == kSplitWaves - 1) {
            Tile<FA> x;
            x.load(c.K_kept, c.V_kept, c.K_scales, c.V_scales, work.begin + work.kept_tiles * T, left, lane);
            take<FA, true>(r, x, q, a.scale_log2, (1u << min(max(left - quarter * (T / 4), 0), 8)) - 1u);
        }
    }
    constexpr int T = Tile<FB>::T;
    const int64_t base = (int64_t)g * c.stride;
    Tile<FB>::queries(q, q_row, quarter);
    // (chunks of the cache follow those of the kept rows)
    stream<FB>(Walk((share + shares - work.kept_chunks % shares) % shares, work.cache_chunks, work.cache_tiles, shares, a.chunk, wave), r, q, a.scale_log2,
               [&](Tile<FB>& x, int64_t tile) { x.load(c.K, c.V, nullptr, nullptr, base + work.row_of((int)tile), T, lane); });
    // (the last share and its last waves first: they have least of the rest)
    for (int i = (shares - 1 - share) * kSplitWaves + kSplitWaves - 1 - wave; i < work.cache_masked; i += shares * kSplitWaves) {
        const int near = i < work.low_masked ? i - (work.seen.first % T != 0) : work.near_end + i - work.low_masked;        // -1: the end of the first rows
        const int j0 = near < 0 ? work.first_tiles * T : work.seen.low + near * T, count = min(T, (near < 0 ? work.seen.first : work.seen.high) - j0);
        const int p = work.seen.p0 + (t - work.t0);
        Tile<FB> x;
        x.load(c.K, c.V, nullptr, nullptr, base + j0, count, lane);
        uint32_t mask = 0;
#pragma unroll
        for (int e = 0; e < T / 4; ++e) {
            const int k = quarter * (T / 4) + e;
            mask |= k < count && sees(p, j0 + k, c.window, c.sinks) ? 1u << e : 0u;
        }
        take<FB, true>(r, x, q, a.scale_log2, mask);
    }

    // the four waves' parts
    r.sum = quarters_sum(r.sum);
    if (quarter == 0) {
        tops[wave][col] = r.top;
        sums[wave][col] = r.sum;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float* to = &part[wave][col][quarter * 32 + j * 8];
        *(f32x4a*)to = (f32x4a){r.o[0][j], r.o[1][j], r.o[2][j], r.o[3][j]};
        *(f32x4a*)(to + 4) = (f32x4a){r.o[4][j], r.o[5][j], r.o[6][j], r.o[7][j]};
    }
    __syncthreads();
    const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 8;
    const int Rw = row_tile * kRowTile + row;
    if (Rw >= a.rows) return;
    float top = tops[0][row], sum = 0.f, o[8] = {};
#pragma unroll
    for (int w = 1; w < kSplitWaves; ++w) top = fmaxf(top, tops[w][row]);
    const float off = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) {
        const float weight = __builtin_amdgcn_exp2f(tops[w][row] - off);
        if (tops[w][row] == -INFINITY) continue;           // (a wave without keys)
        sum += weight * sums[w][row];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] += weight * part[w][row][d0 + i];
    }
    if (a.shares > 1) {
        const int64_t at = ((int64_t)g * a.rows + Rw) * a.shares + share;
        *(f32x4a*)(a.part_o + at * 128 + d0) = (f32x4a){o[0], o[1], o[2], o[3]};
        *(f32x4a*)(a.part_o + at * 128 + d0 + 4) = (f32x4a){o[4], o[5], o[6], o[7]};
        if (d0 == 0) a.part_ml[at] = (f32x2a){top, sum};
        return;
    }
    const float over = top == -INFINITY ? 0.f : 1.f / sum;
    const int tw = Rw / c.group, hw = head * c.group + Rw % c.group;
    const int64_t out_row = ((int64_t)b * c.m + tw) * c.kv * c.group + hw;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = top == -INFINITY ? 0.f : o[i] * over;
    if (FB == kBf16) {
        *(u32x4a*)((char*)c.out + out_row * 256 + d0 * 2) = (u32x4a){pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7])};
    } else {
        *(f32x4a*)((char*)c.out + out_row * 512 + d0 * 4) = (f32x4a){o[0], o[1], o[2], o[3]};
        *(f32x4a*)((char*)c.out + out_row * 512 + d0 * 4 + 16) = (f32x4a){o[4], o[5], o[6], o[7]};
    }
    if (c.lse && d0 == 0) c.lse[((int64_t)b * c.kv * c.group + hw) * c.m + tw] = top == -INFINITY ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Joins the shares of one row: four waves take every fourth share, a lane two channels.
template <int FA, int FB>
__global__ __launch_bounds__(256) void attend_join_kernel(SplitArgs a) {
    __shared__ float part[4][128], sums[4];
    const AttendCall& c = a.c;
    const int g = blockIdx.x / a.rows, R = blockIdx.x % a.rows;
    const Work<FA, FB> work(a, g, R / kRowTile);
    const int shares = work.shares(a);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * a.shares;
    float top = -INFINITY;
    for (int s = lane; s < shares; s += 64) top = fmaxf(top, a.part_ml[at + s].x);
#pragma unroll
    for (int k = 32; k; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float off = top == -INFINITY ? 0.f : top;
    f32x2a o = {0, 0};
    float sum = 0.f;
#pragma unroll 4
    for (int s = wave; s < shares; s += 4) {
        const f32x2a ml = a.part_ml[at + s];
        const f32x2a x = *(const f32x2a*)(a.part_o + (at + s) * 128 + lane * 2);
        const float weight = __builtin_amdgcn_exp2f(ml.x - off);
        sum += weight * ml.y;
        o += weight * x;
    }
    part[wave][lane * 2] = o.x;
    part[wave][lane * 2 + 1] = o.y;
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    sum = sums[0] + sums[1] + sums[2] + sums[3];
    const float over = top == -INFINITY ? 0.f : 1.f / sum;
    float y[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int d = lane * 2 + i;
        y[i] = top == -INFINITY ? 0.f : (part[0][d] + part[1][d] + part[2][d] + part[3][d]) * over;
    }
    const int b = g / c.kv, t = R / c.group, h = (g % c.kv) * c.group + R % c.group;
    const int64_t out_row = ((int64_t)b * c.m + t) * c.kv * c.group + h;
    if (FB == kBf16) ((uint32_t*)c.out)[out_row * 64 + lane] = pack_bf16(y[0], y[1]);
    else ((f32x2a*)c.out)[out_row * 64 + lane] = (f32x2a){y[0], y[1]};
    if (c.lse && lane == 0) c.lse[((int64_t)b * c.kv * c.group + h) * c.m + t] = top == -INFINITY ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int FA, int FB>
hipError_t launch(const SplitArgs& a, hipStream_t stream) {
    const int64_t blocks = (int64_t)a.shares * a.groups * a.row_tiles;
    attend_split_kernel<FA, FB><<<(unsigned)blocks, kSplitWaves * 64, 0, stream>>>(a);
    if (a.shares > 1) attend_join_kernel<FA, FB><<<(unsigned)((int64_t)a.groups * a.rows), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_split(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream) {
    SplitArgs a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.groups = (int)(call.count * call.kv);
    a.rows = call.m * call.group;
    a.row_tiles = (a.rows + kRowTile - 1) / kRowTile;
    // tiles of keys that a head has on average, as far as the host knows
    const bool mx = call.K_scales != nullptr, f32 = call.dtype == CURDKV_DTYPE_F32;
    const int T = f32 ? 16 : 32;
    int64_t keys = call.n;
    if (call.window > 0) keys = min(keys, (int64_t)call.window + call.sinks + call.m);
    const int64_t kept = call.offsets ? (call.rows + a.groups - 1) / a.groups : 0;
    const int64_t tiles = (kept + T - 1) / T + (keys + T - 1) / T;
    const int64_t others = (int64_t)a.groups * a.row_tiles;
    // two workgroups a unit, in chunks of one tile a wave or more; room for heads of four times the average
    const int64_t wanted = max((int64_t)1, (2 * ctx->num_cu + others - 1) / others);
    int64_t chunk = ((tiles + wanted - 1) / wanted + kSplitWaves - 1) / kSplitWaves * kSplitWaves;
    a.chunk = (int)max((int64_t)kSplitWaves, min(chunk, (int64_t)1 << 20));
    const int64_t rooms = call.scratch ? min(kPartRows, call.scratch_bytes / kPartBytes) : 0;
    int64_t shares = call.offsets ? 4 * ((kept + T - 1) / T) / a.chunk + 2 + (keys + T - 1) / T / a.chunk : (tiles + a.chunk - 1) / a.chunk + (call.sinks > 0);
    shares = max((int64_t)1, min(shares, min(4 * wanted, rooms / ((int64_t)a.groups * a.rows))));
    a.shares = (int)shares;
    a.part_o = (float*)call.scratch;
    a.part_ml = (f32x2a*)(a.part_o + (int64_t)a.groups * a.rows * a.shares * 128);
    if (!call.offsets) return f32 ? launch<kNone, kF32>(a, stream) : launch<kNone, kBf16>(a, stream);
    if (mx) return f32 ? launch<kMxF32, kF32>(a, stream) : launch<kMxBf16, kBf16>(a, stream);
    return f32 ? launch<kF32, kF32>(a, stream) : launch<kBf16, kBf16>(a, stream);
}

}  // namespace curdkv
