// Attention of many tokens over an fp32 cache: as attend_prompt.hip, in fp32 products throughout.  Bound by the matrix units: mfma_f32_32x32x2 gives
// 64 flops a clock and SIMD, a sixteenth of bf16, so that the softmax between the products costs nothing worth hiding and a tile of 32 keys is
// taken in one go.
//
// S^T = K Q^T: lane (key or row R = lane % 32, half) has channels 8 s + 4 half + 0..3 of both, four products from one 16-byte read of K.  O^T = V^T P^T:
// product i takes the keys 8 (i / 4) + i % 4 (half 0) and 4 further (half 1), which is where register i of S^T comes from; V is read 16 bytes at a time
// as well, a lane's four channels 4 (lane % 32) + 0..3 going to four products.

#include <type_traits>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

constexpr int kKeys = 32;              // of a tile

struct PromptF32Args {
    AttendCall c;
    float scale_log2;
    int groups, rows, row_tiles;
};

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES / 2) void attend_prompt_f32_kernel(PromptF32Args a) {
    constexpr int kTileRows = WAVES * 32, kBlocks = 16 / WAVES;
    __shared__ __attribute__((aligned(16))) char Ks[2][kKeys * 512], Vs[2][kKeys * 512];
    const AttendCall& c = a.c;
    const int g = blockIdx.x % a.groups, row_tile = a.row_tiles - 1 - blockIdx.x / a.groups;      // long ones first
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int b = g / c.kv, head = g % c.kv;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n;
    const int t_first = row_tile * kTileRows / c.group, t_last = min(c.m - 1, (row_tile * kTileRows + kTileRows - 1) / c.group);
    const Seen seen = seen_rows(length, c.m, t_first, t_last, c.window, c.sinks);
    const int first_tiles = (seen.first + kKeys - 1) / kKeys, tiles = first_tiles + (seen.high - seen.low + kKeys - 1) / kKeys;
    const auto row_of = [&](int tile) { return tile < first_tiles ? tile * kKeys : seen.low + (tile - first_tiles) * kKeys; };
    const auto count_of = [&](int tile) { return min(kKeys, (tile < first_tiles ? seen.first : seen.high) - row_of(tile)); };

    const int R0 = row_tile * kTileRows + wave * 32, R = min(R0 + col, a.rows - 1), t = R / c.group, p = length - c.m + t;
    const int p_first = length - c.m + min(R0, a.rows - 1) / c.group, p_last = length - c.m + min(R0 + 31, a.rows - 1) / c.group;
    const int64_t q_row = (((int64_t)b * c.m + t) * c.kv + head) * c.group + R % c.group;
    f32x4a q[16];
#pragma unroll
    for (int s = 0; s < 16; ++s) q[s] = ((const f32x4a*)((const char*)c.Q + q_row * 512))[2 * s + half];

    const char* Kg = (const char*)c.K + (int64_t)g * c.stride * 512;
    const char* Vg = (const char*)c.V + (int64_t)g * c.stride * 512;
    const uint32_t k_lds = lds_address(&Ks[0][0]), v_lds = lds_address(&Vs[0][0]);
    // Two rows a block of 1 KB; K's 16-byte pieces permuted by row % 8, so that eight rows' reads of one piece meet different banks.
    const auto fetch = [&](int tile) {
        const int64_t j0 = row_of(tile);
        const int count = count_of(tile), piece = lane & 31;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const int block = wave * kBlocks + i, row = block * 2 + half;
            const uint32_t from = min(row, count - 1) * 512, to = (tile & 1) * (kKeys * 512) + block * 1024;
            dma16(k_lds + to, Kg + j0 * 512, from + ((piece ^ (row & 7)) << 4));
            dma16(v_lds + to, Vg + j0 * 512, from + (piece << 4));
        }
    };

    f32x16a o[4];                      // o[j]: channels 4 (row of the product) + j
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
    float top = -INFINITY, sum = 0.f;

    const auto take = [&](auto masked, int tile) {
        constexpr bool MASKED = decltype(masked)::value;
        const char *Kt = Ks[tile & 1] + col * 512, *Vt = Vs[tile & 1];
        f32x16a s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const f32x4a k = *(const f32x4a*)(Kt + (((2 * x + half) ^ (col & 7)) << 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j], q[x][j], s, 0, 0, 0);
        }
        const int j0 = row_of(tile), far = min(p - j0, count_of(tile) - 1) - half * 4, near = (c.window > 0 ? p - j0 - c.window : -1) - half * 4, sink = c.sinks - j0 - half * 4;
        const auto has = [&](int key) { return key <= far && (key > near || key < sink); };
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (MASKED) s[i] = has(i / 4 * 8 + i % 4) ? s[i] : -INFINITY;
            most = fmaxf(most, s[i]);
        }
        most = fmaxf(top, halves_max(most) * a.scale_log2);
        if (__any(most > top)) {
            const float keep = most > top ? __builtin_amdgcn_exp2f(top - most) : 1.f;
            sum *= keep;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] *= keep;
            top = most;
        }
        const float off = MASKED && top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2, -off));
            sum += s[i];
        }
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            f32x4a v = *(const f32x4a*)(Vt + (i / 4 * 8 + half * 4 + i % 4) * 512 + col * 16);
            if constexpr (MASKED) {
                // an infinity or NaN must not meet the zero weight of a row that does not see it: a zero in its place, ..
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool not_finite = (__float_as_uint(v[j]) & 0x7F800000u) == 0x7F800000u;
                    bad |= not_finite;
                    v[j] = not_finite ? 0.f : v[j];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[j], s[i], o[j], 0, 0, 0);
        }
        if (MASKED && __any(bad)) {
            // .. and then they reach the rows that do see them: whatever the weight, an infinity or NaN comes of it.
            for (int key = 0; key < kKeys; ++key) {
                if (!has(key - half * 4)) continue;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const f32x4a v = *(const f32x4a*)(Vt + key * 512 + (i / 4 * 8 + half * 4 + i % 4) * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if ((__float_as_uint(v[j]) & 0x7F800000u) == 0x7F800000u) o[j][i] += v[j];
                }
            }
        }
    };

    if (tiles > 0) {
        fetch(0);
        dma_wait();
    }
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) fetch(tile + 1);
        const int j0 = row_of(tile);
        // (of this wave's tokens) all see all of the tile; none sees any of it
        const bool whole = count_of(tile) == kKeys && j0 + kKeys - 1 <= p_first && (c.window <= 0 || p_last - j0 < c.window || j0 + kKeys <= c.sinks);
        const bool none = j0 > p_last || (c.window > 0 && j0 + kKeys - 1 <= p_first - c.window && j0 >= c.sinks);
        if (whole) take(std::false_type{}, tile);
        else if (!none) take(std::true_type{}, tile);
        dma_wait();
        __syncthreads();
    }

    sum = halves_sum(sum);
    if (R0 + col >= a.rows) return;
    const bool empty = top == -INFINITY;
    const float over = empty ? 0.f : 1.f / sum;
    char* out = (char*)c.out + q_row * 512;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        *(f32x4a*)(out + (i / 4 * 8 + half * 4 + i % 4) * 16) = (f32x4a){o[0][i] * over, o[1][i] * over, o[2][i] * over, o[3][i] * over};
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
    // 128 rows a workgroup where that gives every unit four, 64 below
    if ((int64_t)a.groups * ((a.rows + 127) / 128) >= 4 * (int64_t)ctx->num_cu) return launch(attend_prompt_f32_kernel<4>, 4);
    return launch(attend_prompt_f32_kernel<2>, 2);
}

}  // namespace curdkv
