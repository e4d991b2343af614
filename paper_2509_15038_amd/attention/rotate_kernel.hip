// From a layer's projections to its queries and cache rows: for every head of every new token an optional RMS norm over the
// head's 128 channels, y = x / sqrt(mean x^2 + eps) * w, and the rotation by position,
//     (a, b) -> (a cos - b sin, b cos + a sin)
// for the channel pairs (i, i + 64) or (2 i, 2 i + 1); keys and values go to their rows of the cache, transposed from the
// projections' token-major order to the cache's head-major one on the way.
//
// HBM-bound: every row is read and written once.  Eight lanes take a row, 16 channels a lane: those of eight whole pairs in
// either pairing, so that the rotation is in-lane and the norm needs three exchanges.  The eight lanes stay with their token and
// take several of its heads, so that cosines and sines (512 bytes a token, twice a bf16 row) are read once for all of them.
// Everything between load and store is in 32 bits; the store is the one rounding.
// Measured: 32768 tokens of 32 + 8 + 8 heads with norms (822 MB) 140 us, 5.9 TB/s; one token of 4 sequences 4.0 to 4.7 us a call, the
// kernel 3.5.  fp32, 32768 tokens (1628 MB) 444 us, 3.7 TB/s: a lane's 32 bytes go as two stores of 16, whose half lines past the caches are 1.5 times the bytes.

#include <algorithm>

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

struct RotateArgs {
    const char* qkv;
    int64_t m, tokens, row_stride;     // row_stride in bytes
    const int32_t *starts, *positions;
    const float* table;
    int64_t table_rows;
    const void *q_weight, *k_weight;
    float eps;
    int kv, group;
    char *Q, *K, *V;
    int64_t stride;
    int64_t first;                     // a launch's first token
};

template <int CTRL>
__device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true)); }
// sum over groups of eight lanes: quad_perm xor 1, xor 2, then the mirror of a half row
__device__ __forceinline__ float eights_sum(float x) {
    x += dpp<0xB1>(x);
    x += dpp<0x4E>(x);
    x += dpp<0x141>(x);
    return x;
}

template <bool BF16>
struct Sixteen {                       // 16 channels of a row: a lane's two pieces of eight
    u32x4a raw[BF16 ? 2 : 4];
    template <bool PAST>
    __device__ __forceinline__ void load(const char* row, int first, int second) {
        constexpr int W = BF16 ? 1 : 2;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const u32x4a *x = (const u32x4a*)row + first * W + i, *y = (const u32x4a*)row + second * W + i;
            raw[i] = PAST ? __builtin_nontemporal_load(x) : *x;
            raw[W + i] = PAST ? __builtin_nontemporal_load(y) : *y;
        }
    }
    template <bool PAST>
    __device__ __forceinline__ void store(char* row, int first, int second) const {
        constexpr int W = BF16 ? 1 : 2;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            u32x4a *x = (u32x4a*)row + first * W + i, *y = (u32x4a*)row + second * W + i;
            if (PAST) __builtin_nontemporal_store(raw[i], x), __builtin_nontemporal_store(raw[W + i], y);
            else *x = raw[i], *y = raw[W + i];
        }
    }
    __device__ __forceinline__ void get(float* x) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (BF16) {
                const uint32_t w = raw[i / 8][(i % 8) / 2];
                x[i] = __uint_as_float(i % 2 ? w & 0xFFFF0000u : w << 16);
            } else {
                x[i] = __uint_as_float(raw[i / 4][i % 4]);
            }
        }
    }
    __device__ __forceinline__ void set(const float* x) {
#pragma unroll
        for (int i = 0; i < (BF16 ? 8 : 16); ++i) {
            if (BF16) raw[i / 4][i % 4] = pack_bf16(x[2 * i], x[2 * i + 1]);
            else raw[i / 4][i % 4] = __float_as_uint(x[i]);
        }
    }
};

// TOKENS a workgroup; PAIRS: neighbours rotate together; PAST: rows pass the caches.  A lane u of eight holds pairs 8 u .. 8 u + 7.
template <bool BF16, bool PAIRS, int TOKENS, bool PAST>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a) {
    constexpr int kSlots = 32 / TOKENS, kRow = BF16 ? 256 : 512;
    const int u = threadIdx.x & 7, slot = threadIdx.x >> 3;
    const int64_t token = a.first + (int64_t)blockIdx.x * TOKENS + slot / kSlots;
    if (token >= a.tokens) return;
    const int64_t b = token / a.m, i = token - b * a.m;
    const int first = PAIRS ? 2 * u : u, second = PAIRS ? 2 * u + 1 : u + 8;       // pieces of eight channels
    const int64_t start = a.starts ? a.starts[b] : 0, at = start + i;
    int64_t position = a.positions ? a.positions[token] : at;
    position = position < 0 ? 0 : position < a.table_rows ? position : a.table_rows - 1;
    const float* turn = a.table + position * 128 + u * 8;
    float cosine[8], sine[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        *(f32x4a*)&cosine[4 * k] = *(const f32x4a*)(turn + 4 * k);
        *(f32x4a*)&sine[4 * k] = *(const f32x4a*)(turn + 64 + 4 * k);
    }
    const bool in_cache = at >= 0 && at < a.stride;
    const int queries = a.kv * a.group, heads = queries + 2 * a.kv;
    const char* rows = a.qkv + token * a.row_stride;
    for (int h = slot % kSlots; h < heads; h += kSlots) {
        Sixteen<BF16> x;
        x.template load<PAST>(rows + (int64_t)h * kRow, first, second);
        if (h < queries + a.kv) {
            float y[16], z[16];
            x.get(y);
            const void* weight = h < queries ? a.q_weight : a.k_weight;
            if (weight) {
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < 16; ++k) sum += y[k] * y[k];
                const float over = 1.f / sqrtf(eights_sum(sum) * (1.f / 128.f) + a.eps);
                Sixteen<BF16> w;
                w.template load<false>((const char*)weight, first, second);
                w.get(z);
#pragma unroll
                for (int k = 0; k < 16; ++k) y[k] = y[k] * over * z[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int p = PAIRS ? 2 * k : k, q = PAIRS ? 2 * k + 1 : k + 8;
                z[p] = y[p] * cosine[k] - y[q] * sine[k];
                z[q] = y[q] * cosine[k] + y[p] * sine[k];
            }
            x.set(z);
        }
        if (h < queries) {
            x.template store<PAST>(a.Q + (token * queries + h) * kRow, first, second);
        } else if (in_cache) {
            const int head = h - queries < a.kv ? h - queries : h - queries - a.kv;
            x.template store<PAST>((h - queries < a.kv ? a.K : a.V) + ((b * a.kv + head) * a.stride + at) * kRow, first, second);
        }
    }
}

template <bool BF16, bool PAIRS>
hipError_t launch(const curdkv_ctx* ctx, RotateArgs a, hipStream_t stream) {
    // Four tokens a workgroup where that still gives every unit four; one, its heads over all lanes, below.  Rows that the caches would not hold until
    // they are read again pass them by (32768 tokens of 48 heads: 159 us, 144 so).
    const int64_t bytes = a.tokens * a.kv * (a.group + 2) * (BF16 ? 512 : 1024);
    if (a.tokens < 16 * (int64_t)ctx->num_cu) {
        rotate_kernel<BF16, PAIRS, 1, false><<<(unsigned)a.tokens, 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    // (a launch's threads are counted in 32 bits: 2^25 tokens each)
    for (; a.first < a.tokens; a.first += 1 << 25) {
        const unsigned blocks = (unsigned)((std::min(a.tokens - a.first, (int64_t)1 << 25) + 3) / 4);
        if (bytes <= kPastCaches) rotate_kernel<BF16, PAIRS, 4, false><<<blocks, 256, 0, stream>>>(a);
        else rotate_kernel<BF16, PAIRS, 4, true><<<blocks, 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride, const int32_t* starts,
                         const int32_t* positions, const float* table, int64_t table_rows, const void* q_weight, const void* k_weight,
                         float eps, bool pairs, void* Q, void* K, void* V, int64_t stride, hipStream_t stream) {
    const bool bf16 = ctx->cfg.dtype == CURDKV_DTYPE_BF16;
    const RotateArgs a{(const char*)qkv, m, count * m, row_stride * (bf16 ? 2 : 4), starts, positions, table, table_rows, q_weight, k_weight, eps,
                       ctx->cfg.kv_heads, ctx->cfg.group_size, (char*)Q, (char*)K, (char*)V, stride, 0};
    if (bf16) return pairs ? launch<true, true>(ctx, a, stream) : launch<true, false>(ctx, a, stream);
    return pairs ? launch<false, true>(ctx, a, stream) : launch<false, false>(ctx, a, stream);
}

}  // namespace curdkv
