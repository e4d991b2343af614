// Attention of many tokens (prompts) over a bf16 cache: tiles of 64 keys against 32 rows R a wave, the softmax's maximum and sum running
// along.  Bound by the matrix units and the exponentials: 4 * 128 flops and one exponential for a visible (row, key).
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
// maximum passes it by more, so that most tiles scale nothing.

#include <type_traits>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

typedef float f32x16a __attribute__((ext_vector_type(16)));
typedef short s16x4a __attribute__((ext_vector_type(4)));

constexpr int kKeys = 64;              // of a tile
constexpr float kLoose = 8.f;

struct PromptArgs {
    AttendCall c;
    float scale_log2;
    int groups, rows, row_tiles;
};

__device__ __forceinline__ u32x2 read_transposed(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4a*)p));
}
__device__ __forceinline__ float halves_max(float x) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float halves_sum(float x) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}
// 64 lanes' 16 bytes from base + at to LDS from `to` on, in order of the lanes.  Nothing waits for it but dma_wait().
__device__ __forceinline__ void dma16(uint32_t to, const void* base, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory");
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_prompt_kernel(PromptArgs a) {
    constexpr int kStage = 16 / WAVES, kTileRows = WAVES * 32;
    __shared__ __attribute__((aligned(16))) char Ks[2][kKeys * 256], Vs[2][kKeys * 256];
    const AttendCall& c = a.c;
    const int g = blockIdx.x % a.groups, row_tile = a.row_tiles - 1 - blockIdx.x / a.groups;      // long ones first
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int b = g / c.kv, head = g % c.kv;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n;

    const int t_first = row_tile * kTileRows / c.group, t_last = min(c.m - 1, (row_tile * kTileRows + kTileRows - 1) / c.group);
    const Seen seen = seen_rows(length, c.m, t_first, t_last, c.window, c.sinks);
    const int first_tiles = (seen.first + kKeys - 1) / kKeys, tiles = first_tiles + (seen.high - seen.low + kKeys - 1) / kKeys;
    const auto row_of = [&](int tile) { return tile < first_tiles ? tile * kKeys : seen.low + (tile - first_tiles) * kKeys; };
    const auto count_of = [&](int tile) { return min(kKeys, (tile < first_tiles ? seen.first : seen.high) - row_of(tile)); };

    // this wave's rows
    const int R0 = row_tile * kTileRows + wave * 32;
    const int w_first = min(R0, a.rows - 1) / c.group, w_last = min(R0 + 31, a.rows - 1) / c.group;
    const int p_first = length - c.m + w_first, p_last = length - c.m + w_last;
    const int R = min(R0 + col, a.rows - 1), t = R / c.group, p = length - c.m + t;
    const int64_t q_row = (((int64_t)b * c.m + t) * c.kv + head) * c.group + R % c.group;
    u32x4a q[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = ((const u32x4a*)((const char*)c.Q + q_row * 256))[2 * s + half];

    const char* Kg = (const char*)c.K + (int64_t)g * c.stride * 256;
    const char* Vg = (const char*)c.V + (int64_t)g * c.stride * 256;
    // A tile's 1 KB blocks of 16 rows' columns: this wave's share.
    const uint32_t k_lds = lds_address(&Ks[0][0]), v_lds = lds_address(&Vs[0][0]);
    const int d_row = lane >> 2, d_piece = lane & 3;
    const auto fetch = [&](int tile, int buffer) {
        const int64_t j0 = row_of(tile);
        const int count = count_of(tile);
#pragma unroll
        for (int i = 0; i < kStage; ++i) {
            const int block = wave * kStage + i, column = block >> 2, row0 = (block & 3) * 16;
            const uint32_t row = min(row0 + d_row, count - 1) * 256 + column * 64, to = buffer * (kKeys * 256) + block * 1024;
            dma16(k_lds + to, Kg + j0 * 256, row + ((d_piece ^ ((d_row >> 1) & 3)) << 4));
            dma16(v_lds + to, Vg + j0 * 256, row + (d_piece << 4));
        }
    };

    // this lane's operands within a tile: K row col, piece 2 x + half; V rows 4 half + lane16 / 4 (+ 8), channels 32 db + ..
    const int l16 = lane & 15, dhalf = (lane >> 4) & 1;
    const int k_at[2] = {col * 64 + ((half ^ ((col >> 1) & 3)) << 4), col * 64 + (((2 + half) ^ ((col >> 1) & 3)) << 4)};
    const int v_at = (4 * half + l16 / 4) * 64 + dhalf * 32 + (l16 & 3) * 8;

    f32x16a o[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float ref = -INFINITY, sum = 0.f;

    // One tile into the running softmax; MASKED: some of this wave's tokens do not see all of it.
    const auto take = [&](auto masked, int buffer, int j0, int count) {
        constexpr bool MASKED = decltype(masked)::value;
        const char *Kt = Ks[buffer], *Vt = Vs[buffer];
        f32x16a s[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const u32x4a k = *(const u32x4a*)(Kt + k_at[x & 1] + (x >> 1) * 4096 + kb * 2048);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, k), __builtin_bit_cast(bf16x8a, q[x]), s[kb], 0, 0, 0);
            }
        }
        // keys of the tile that this row sees: near < key <= far, and those below `sink`
        const int far = min(p - j0, count - 1) - half * 4, near = (c.window > 0 ? p - j0 - c.window : -1) - half * 4, sink = c.sinks - j0 - half * 4;
        if constexpr (MASKED) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = kb * 32 + i / 4 * 8 + i % 4;
                    s[kb][i] = key <= far && (key > near || key < sink) ? s[kb][i] : -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
        top = halves_max(top) * a.scale_log2;
        if (__any(top > ref + kLoose)) {
            const float next = top > ref + kLoose ? top : ref;
            const float keep = next == ref ? 1.f : __builtin_amdgcn_exp2f(ref - next);
            sum *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db) o[db] *= keep;
            ref = next;
        }
        const float off = MASKED && ref == -INFINITY ? 0.f : ref;
        uint32_t pb[16];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], a.scale_log2, -off));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i + 1], a.scale_log2, -off));
                sum += x + y;
                pb[kb * 8 + i / 2] = pack_bf16(x, y);
            }
        bool bad = false;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const u32x4a pu = {pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]};
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const u32x2 x = read_transposed(Vt + v_at + db * 4096 + u * 1024);
                const u32x2 y = read_transposed(Vt + v_at + db * 4096 + u * 1024 + 512);
                u32x4a v = {x.x, x.y, y.x, y.y};
                if constexpr (MASKED) {
                    // an infinity or NaN must not meet the zero weight of a row that does not see it
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const bool low = (v[w] & 0x7F80u) == 0x7F80u, high = (v[w] & 0x7F800000u) == 0x7F800000u;
                        bad |= low || high;
                        v[w] &= (low ? 0xFFFF0000u : ~0u) & (high ? 0x0000FFFFu : ~0u);
                    }
                }
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8a, v), __builtin_bit_cast(bf16x8a, pu), o[db], 0, 0, 0);
            }
        }
        if (MASKED && __any(bad)) {
            // They reach the rows that do see them: whatever the weight, an infinity or NaN comes of it.
            for (int key = 0; key < kKeys; ++key) {
                const int k = key - half * 4;
                if (!(k <= far && (k > near || k < sink))) continue;
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
    };

    if (tiles > 0) {
        fetch(0, 0);
        dma_wait();
    }
    __syncthreads();
    // Tiles that all of the workgroup's tokens see all of, in the middle, have a loop of their own: the accumulators then stay where they are.
    const int whole_end = first_tiles + max(0, (min(seen.high, seen.p0 + 1) - seen.low) / kKeys);
    const int hidden = c.window > 0 ? max(0, seen.p1 - c.window + 1 - seen.low) : 0;             // rows from `low` on that the last token does not see
    const int whole_begin = min(first_tiles + (hidden + kKeys - 1) / kKeys, whole_end);
    int tile = 0;
    for (int part = 0; part < 3; ++part) {
        if (part == 1) {
            for (; tile < whole_end; ++tile) {
                if (tile + 1 < tiles) fetch(tile + 1, (tile & 1) ^ 1);
                take(std::false_type{}, tile & 1, row_of(tile), kKeys);
                dma_wait();
                __syncthreads();
            }
        } else {
            const int end = part == 0 ? whole_begin : tiles;
            for (; tile < end; ++tile) {
                if (tile + 1 < tiles) fetch(tile + 1, (tile & 1) ^ 1);
                const int j0 = row_of(tile);
                // (none of this wave's tokens sees any of it)
                const bool none = j0 > p_last || (c.window > 0 && j0 + kKeys - 1 <= p_first - c.window && j0 >= c.sinks);
                if (!none) take(std::true_type{}, tile & 1, j0, count_of(tile));
                dma_wait();
                __syncthreads();
            }
        }
    }

    sum = halves_sum(sum);
    if (R0 + col >= a.rows) return;
    const bool empty = ref == -INFINITY;
    const float over = empty ? 0.f : 1.f / sum;
    char* out = (char*)c.out + q_row * 256;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x2 x = {pack_bf16(o[db][4 * i] * over, o[db][4 * i + 1] * over), pack_bf16(o[db][4 * i + 2] * over, o[db][4 * i + 3] * over)};
            *(u32x2*)(out + (db * 32 + i * 8 + half * 4) * 2) = x;
        }
    if (c.lse && half == 0) c.lse[((int64_t)b * c.kv * c.group + head * c.group + R % c.group) * c.m + t] = empty ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

hipError_t launch_attend_prompt(const curdkv_ctx*, const AttendCall& call, hipStream_t stream) {
    constexpr int kWaves = 4;
    PromptArgs a;
    a.c = call;
    a.scale_log2 = call.scale * (1.f / kLn2);
    a.groups = (int)(call.count * call.kv);
    a.rows = call.m * call.group;
    a.row_tiles = (a.rows + kWaves * 32 - 1) / (kWaves * 32);
    attend_prompt_kernel<kWaves><<<(unsigned)((int64_t)a.groups * a.row_tiles), kWaves * 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace curdkv
