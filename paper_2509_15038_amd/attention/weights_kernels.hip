// The attention weight that every key of a cache got from a sequence's last m tokens, summed over them and the query heads of its KV head:
//     mass[j] = decay mass[j] + sum over rows R = (token, head) that see j of exp(scale q_R.k_j - lse_R),
// lse_R being the logarithm of the row's softmax denominator, which the attention has written.  With it no maximum has to be found: every weight is at
// most 1 (as far as lse is what the scores make it), and a key's sum is its own affair: one wave's, in a fixed order, without atomics.
// S = Q K^T: 16 rows R are the A operand of mfma_f32_16x16x32_bf16 (16x16x4 for fp32), 16 keys the B operand, so that a lane holds four rows' scores of
// one key, and adds their weights up in a register until all rows are through.

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

struct WeightsArgs {
    WeightsCall c;
    float scale_log2;
    int rows, key_tiles;               // m * group; workgroups of 64 keys a head
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

template <bool BF16>
__global__ __launch_bounds__(256) void weights_kernel(WeightsArgs a) {
    constexpr int kRow = BF16 ? 256 : 512;
    const WeightsCall& c = a.c;
    const int g = blockIdx.x / a.key_tiles, b = g / c.kv, head = g % c.kv;
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    const int j0 = (blockIdx.x % a.key_tiles * 4 + (threadIdx.x >> 6)) * 16;
    const int length = c.lengths ? min(max(c.lengths[b], 0), c.n) : c.n;
    if (j0 >= length) return;
    const int j = j0 + col, j1 = min(j0 + 15, length - 1);
    Operand<BF16> k, q;
    k.load((const char*)c.K + ((int64_t)g * c.stride + min(j, length - 1)) * kRow, quarter);
    const Tokens t = tokens_that_see(length, c.m, j0, j1, c.window, c.sinks);
    float sum = 0.f;
    for (int R0 = t.first * c.group & ~15; R0 < (t.last + 1) * c.group; R0 += 16) {
        const auto row_of = [&](int R) { return (((int64_t)b * c.m + R / c.group) * c.kv + head) * c.group + R % c.group; };
        q.load((const char*)c.Q + row_of(min(R0 + col, a.rows - 1)) * kRow, quarter);
        const f32x4a s = Operand<BF16>::product(q, k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int R = R0 + 4 * quarter + i, at = min(R, a.rows - 1), token = at / c.group;
            const float lse = c.lse[((int64_t)b * c.kv * c.group + head * c.group + at % c.group) * c.m + token];
            const bool seen = R < a.rows && j < length && lse != -INFINITY && sees(length - c.m + token, j, c.window, c.sinks);
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2, -lse * (1.f / kLn2)));
            sum += seen ? w : 0.f;
        }
    }
    sum = quarters_sum(sum);
    if (quarter == 0 && j < length) {
        float* to = c.mass + (int64_t)g * c.mass_stride + j;
        *to = c.decay == 0.f ? sum : __builtin_fmaf(c.decay, *to, sum);
    }
}

}  // namespace

hipError_t launch_weights(const curdkv_ctx* ctx, const WeightsCall& call, hipStream_t stream) {
    WeightsArgs a{call, call.scale * (1.f / kLn2), call.m * call.group, (call.n + 63) / 64};
    const unsigned blocks = (unsigned)(call.count * call.kv * a.key_tiles);
    if (call.dtype == CURDKV_DTYPE_BF16) weights_kernel<true><<<blocks, 256, 0, stream>>>(a);
    else weights_kernel<false><<<blocks, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace curdkv
