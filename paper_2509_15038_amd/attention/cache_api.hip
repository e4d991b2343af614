// C ABI of the operators that keep a cache at its size and let sequences share one: argument checks and launches (rotate_kernel.hip, weights_kernels.hip,
// evict_kernels.hip, attend_shared.hip).

#include <algorithm>
#include <cmath>

#include "attend_internal.h"

using namespace curdkv;

namespace {

int run_shared(curdkv_ctx* ctx, const void* Q, const void* K_kept, const void* V_kept, const uint8_t* K_scales, const uint8_t* V_scales,
               const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride,
               const int32_t* tail_lengths, int64_t count, int64_t share, int64_t m, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes, void* stream) {
    AttendCall c;
    const int rc = check_kept(ctx, &c, Q, K_kept, V_kept, K_scales, V_scales, offsets, total, rows, K_tail, V_tail, tail_n, tail_stride, tail_lengths, count, share, m,
                              scale, out, lse, scratch, scratch_bytes);
    if (rc != CURDKV_OK) return rc;
    if (!scratch || scratch_bytes < CURDKV_ATTEND_SCRATCH_BYTES) return CURDKV_ERR_INVALID_ARG;
    // (the partial results of one token of all heads lie in scratch together, those of a head's kept rows in tiles that are less than half empty: 3 * 2^14 rows of the 73728 that there are)
    if (c.kv > 1 << 10 || (int64_t)c.kv * c.group > 1 << 14) return CURDKV_ERR_UNSUPPORTED;
    return launch_attend_shared(ctx, c, (int)share, (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
}

}  // namespace

extern "C" {

int curdkv_rotate_axes(curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride, const int32_t* starts,
                       const int32_t* positions, int32_t axes, const uint8_t* axis_of, const float* table, int64_t table_rows, const void* q_weight,
                       const void* k_weight, float eps, int32_t pairs, void* Q, void* K, void* V, int64_t stride, void* stream) {
    const int rc = check_rotate(ctx, qkv, count, m, row_stride, table, table_rows, q_weight, k_weight, eps, pairs, Q, K, V, stride);
    if (rc != CURDKV_OK) return rc;
    if (!positions || !axis_of || axes < 1 || axes > 4) return CURDKV_ERR_INVALID_ARG;
    for (int i = 0; i < kHeadDim / 2; ++i)
        if (axis_of[i] >= axes) return CURDKV_ERR_INVALID_ARG;
    return launch_rotate(ctx, qkv, count, m, row_stride, starts, positions, axis_of, table, table_rows, q_weight, k_weight, eps, pairs == 1, Q, K, V, stride,
                         (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
}

int curdkv_attend_weights(curdkv_ctx* ctx, const void* Q, const void* K, const float* lse, int64_t count, int64_t m, int64_t n, int64_t stride,
                          const int32_t* lengths, int64_t window, int32_t n_sink, float scale, float decay, float* mass, int64_t mass_stride, void* scratch,
                          int64_t scratch_bytes, void* stream) {
    const int rc = check_attend(ctx, Q, Q, count, m, n, stride, scale, scratch, scratch_bytes);
    if (rc != CURDKV_OK) return rc;
    if (!K || !lse || !mass || n < 1 || m > ctx->cfg.max_tokens || window < 0 || n_sink < 0 || mass_stride < n || !aligned16({K})) return CURDKV_ERR_INVALID_ARG;
    if (!(decay >= 0.f) || !std::isfinite(decay)) return CURDKV_ERR_INVALID_ARG;
    if ((n + 63) / 64 > kMostBlocks / (count * ctx->cfg.kv_heads)) return CURDKV_ERR_UNSUPPORTED;      // (workgroups of a launch)
    if (ctx->cfg.kv_heads > 1 << 14 || (int64_t)ctx->cfg.kv_heads * ctx->cfg.group_size > 1 << 20) return CURDKV_ERR_UNSUPPORTED;      // (offsets among a few tokens' queries have 32 bits)
    WeightsCall c{};
    c.Q = Q, c.K = K, c.lse = lse, c.count = count, c.stride = stride;
    c.kv = ctx->cfg.kv_heads, c.group = ctx->cfg.group_size, c.m = (int)m, c.n = (int)n, c.dtype = ctx->cfg.dtype;
    c.window = window < n ? (int)window : 0, c.sinks = (int)std::min<int64_t>(n_sink, n);              // (a window of n tokens hides nothing)
    c.lengths = lengths, c.scale = scale, c.decay = decay, c.mass = mass, c.mass_stride = mass_stride;
    c.scratch = scratch, c.scratch_bytes = scratch_bytes;
    return launch_weights(ctx, c, (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
}

int curdkv_evict(curdkv_ctx* ctx, const void* K, const void* V, const float* mass, const int32_t* positions, int64_t count, int64_t n, int64_t stride,
                 const int32_t* lengths, int64_t keep, int32_t n_sink, int64_t recent, void* K_out, void* V_out, float* mass_out, int32_t* positions_out,
                 int64_t out_stride, int32_t* rows, void* stream) {
    if (!ctx || !K || !V || !mass || !K_out || !V_out || !rows) return CURDKV_ERR_INVALID_ARG;
    if (!on_device_of(ctx)) return CURDKV_ERR_INVALID_ARG;
    if (count < 1 || n < 1 || n > ctx->cfg.max_tokens || stride < n || keep < 1 || out_stride < std::min(keep, n)) return CURDKV_ERR_INVALID_ARG;
    if (n_sink < 0 || recent < 0 || recent > keep || n_sink > keep - recent) return CURDKV_ERR_INVALID_ARG;
    if ((K_out == K) != (V_out == V) || K_out == V || V_out == K || K_out == V_out) return CURDKV_ERR_INVALID_ARG;
    if ((K_out == K || mass_out == mass || (positions && positions_out == positions)) && out_stride != stride) return CURDKV_ERR_INVALID_ARG;
    if (!aligned16({K, V, K_out, V_out})) return CURDKV_ERR_INVALID_ARG;
    const int64_t heads = (int64_t)ctx->cfg.kv_heads;
    if (n > kEvictMostRows || keep > 1LL << 30 || count > (1 << 20) / heads) return CURDKV_ERR_UNSUPPORTED;
    EvictCall c{};
    c.K = (const char*)K, c.V = (const char*)V, c.mass = mass, c.positions = positions, c.lengths = lengths;
    c.count = count, c.stride = stride, c.out_stride = out_stride, c.recent = recent;
    c.kv = ctx->cfg.kv_heads, c.n = (int)n, c.keep = (int)keep, c.sinks = n_sink, c.dtype = ctx->cfg.dtype;
    c.K_out = (char*)K_out, c.V_out = (char*)V_out, c.mass_out = mass_out, c.positions_out = positions_out, c.rows = rows;
    return launch_evict(ctx, c, (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
}

int curdkv_attend_shared(curdkv_ctx* ctx, const void* Q, const void* K_kept, const void* V_kept, const int64_t* offsets, int64_t total, int64_t rows,
                         const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride, const int32_t* tail_lengths, int64_t count, int64_t share,
                         int64_t m, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes, void* stream) {
    return run_shared(ctx, Q, K_kept, V_kept, nullptr, nullptr, offsets, total, rows, K_tail, V_tail, tail_n, tail_stride, tail_lengths, count, share, m, scale, out,
                      lse, scratch, scratch_bytes, stream);
}

int curdkv_attend_shared_mx(curdkv_ctx* ctx, const void* Q, const uint8_t* K_codes, const uint8_t* K_scales, const uint8_t* V_codes, const uint8_t* V_scales,
                            const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride,
                            const int32_t* tail_lengths, int64_t count, int64_t share, int64_t m, float scale, void* out, float* lse, void* scratch,
                            int64_t scratch_bytes, void* stream) {
    if (total > 0 && (!K_scales || !V_scales)) return CURDKV_ERR_INVALID_ARG;
    // (nothing kept: the scales are not looked at)
    return run_shared(ctx, Q, K_codes, V_codes, K_scales, V_scales, offsets, total, rows, K_tail, V_tail, tail_n, tail_stride, tail_lengths, count, share, m, scale,
                      out, lse, scratch, scratch_bytes, stream);
}

}  // extern "C"
