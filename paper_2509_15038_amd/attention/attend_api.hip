// C ABI of the operators around a compressed cache: argument checks and launches (rotate_kernel.hip, mx_kernels.hip, attend_split.hip, attend_prompt.hip,
// attend_prompt_f32.hip).

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "attend_internal.h"

using namespace curdkv;

namespace {

// Tiles of 16 rows, and these times the keys, from which the prompts' kernel is the faster one (run_attend).
constexpr int64_t kPromptItems = 600, kPromptProducts = 400000;

}  // namespace

namespace curdkv {

int check_attend(const curdkv_ctx* ctx, const void* Q, const void* out, int64_t count, int64_t m, int64_t n, int64_t stride, float scale,
                 const void* scratch, int64_t scratch_bytes) {
    if (!ctx || !Q || !out) return CURDKV_ERR_INVALID_ARG;
    if (!on_device_of(ctx)) return CURDKV_ERR_INVALID_ARG;
    if (count < 1 || m < 1 || n < 0 || n > ctx->cfg.max_tokens || stride < n) return CURDKV_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale)) return CURDKV_ERR_INVALID_ARG;
    if (scratch_bytes < 0 || !aligned16({Q, out, scratch})) return CURDKV_ERR_INVALID_ARG;
    const int64_t most = (1LL << 31) - 1, heads = (int64_t)ctx->cfg.kv_heads * ctx->cfg.group_size;
    if (count > most / heads || m > most / (count * heads)) return CURDKV_ERR_UNSUPPORTED;     // (grids and row counts are 32 bits)
    return CURDKV_OK;
}

int check_kept(const curdkv_ctx* ctx, AttendCall* to, const void* Q, const void* K_kept, const void* V_kept, const uint8_t* K_scales, const uint8_t* V_scales,
               const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride,
               const int32_t* tail_lengths, int64_t count, int64_t share, int64_t m, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes) {
    if (count < 1 || share < 1) return CURDKV_ERR_INVALID_ARG;
    const int64_t most = 1LL << 31, sequences = share <= most / count ? count * share : most;      // (as many are too many, which is said once all else is right)
    const int rc = check_attend(ctx, Q, out, sequences, m, tail_n, tail_stride, scale, scratch, scratch_bytes);
    if (rc != CURDKV_OK) return rc;
    if (!offsets || total < 0 || rows < 0 || rows > total || (total > 0 && (!K_kept || !V_kept)) || (tail_n > 0 && (!K_tail || !V_tail))) return CURDKV_ERR_INVALID_ARG;
    if (!aligned16({K_kept, V_kept, K_tail, V_tail})) return CURDKV_ERR_INVALID_ARG;
    if (total > (1LL << 31) - 1) return CURDKV_ERR_UNSUPPORTED;        // (a head's rows are counted in 32 bits)
    AttendCall& c = *to;
    c = AttendCall{};
    c.Q = Q, c.out = out, c.lse = lse, c.count = count;
    c.kv = ctx->cfg.kv_heads, c.group = ctx->cfg.group_size, c.m = (int)m, c.dtype = ctx->cfg.dtype, c.scale = scale;
    c.K = K_tail, c.V = V_tail, c.stride = tail_stride, c.lengths = tail_lengths, c.n = (int)tail_n;
    c.offsets = offsets, c.K_kept = K_kept, c.V_kept = V_kept, c.K_scales = K_scales, c.V_scales = V_scales, c.total = total, c.rows = rows;
    c.scratch = scratch, c.scratch_bytes = scratch_bytes;
    return CURDKV_OK;
}

int check_rotate(const curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride, const float* table, int64_t table_rows,
                 const void* q_weight, const void* k_weight, float eps, int32_t pairs, const void* Q, const void* K, const void* V, int64_t stride) {
    if (!ctx || !qkv || !table || !Q || !K || !V) return CURDKV_ERR_INVALID_ARG;
    if (!on_device_of(ctx)) return CURDKV_ERR_INVALID_ARG;
    const int64_t heads = (int64_t)ctx->cfg.kv_heads * (ctx->cfg.group_size + 2LL), bytes = ctx->cfg.dtype == CURDKV_DTYPE_BF16 ? 2 : 4;
    if (count < 1 || m < 1 || stride < 1 || stride > ctx->cfg.max_tokens || table_rows < 1 || row_stride < heads * kHeadDim) return CURDKV_ERR_INVALID_ARG;
    if (pairs != 0 && pairs != 1) return CURDKV_ERR_INVALID_ARG;
    if ((q_weight || k_weight) && (!(eps >= 0.f) || !std::isfinite(eps))) return CURDKV_ERR_INVALID_ARG;
    if (!aligned16({qkv, table, q_weight, k_weight, Q, K, V}) || row_stride * bytes % 16) return CURDKV_ERR_INVALID_ARG;
    if (m > ((1LL << 31) - 1) / count || heads > (1 << 20)) return CURDKV_ERR_UNSUPPORTED;
    return CURDKV_OK;
}

}  // namespace curdkv

namespace {

int run_attend(const curdkv_ctx* ctx, const AttendCall& call, void* stream) {
    // Which kernel: the split one takes tiles of 16 rows (tokens times query heads of a KV head), each of which reads the cache, the prompts' ones 128.
    // bf16, us, split and prompt, 8 heads of 4 a sequence: 9 tokens over 500 rows 9 and 15, over 8000 25 and 25, 32 over 8000 30 and 27; 8 sequences of 9 over 2000 23 and 24, of
    // 16 27 and 25, of 9 over 8000 77 and 50; 32 of 9 over 500 23 and 17, of 8 over 500 15 and 17, over 2000 57 and 50; prompts of 200 tokens 9.5 and 11.2, 300 14.2 and 13.5; 8 of
    // up to 64 12 and 9.  One tile of 16 a head: 32 sequences of 4 tokens over 8000 100 and 164.
    // fp32: prompts of 8 heads 600 tokens 65 and 69, 800 93 and 89, 2400 572 and 344; 64 tokens of 4 sequences over 500 rows 32 and 61, of 16 116 and 65.  Up to two tiles of 16 rows a
    // head the split one always: 256 heads over 4000 rows, 4 rows of a head 159 and 418, 32 309 and 432, 48 460 and 442; 512 over 250 27 and 65, 52 and 66, 72 and 68.
    const int64_t rows = (int64_t)call.m * call.group, heads = call.count * call.kv, items = heads * ((rows + 15) / 16), tiles = heads * ((rows + 127) / 128);
    const int64_t keys = (call.window > 0 ? std::min((int64_t)call.n, (int64_t)call.window + call.sinks + call.m) : call.n) + call.rows / heads;
    const bool f32 = call.dtype == CURDKV_DTYPE_F32;
    // Kept rows in bf16: workgroups do not share out heads of uneven lengths there, which costs more the fewer rows a tile of 128 has: 64 tokens over 3276 rows of 8 uneven heads 41 and
    // 44, 200 92 and 61, 1000 301 and 195 (even heads 4 sequences of 300 103, uneven ones 281); 32 sequences of 6 over 3000 135 and 302.
    const bool prompt = call.offsets ? !call.K_scales && !f32 && rows >= 256 && (items > kPromptItems || items * keys > 2 * kPromptProducts)
                        : f32 ? rows > 32 && 3 * tiles >= 2 * (int64_t)ctx->num_cu : rows > 16 && (items > kPromptItems || items * keys > kPromptProducts);
    const auto launch = !prompt ? launch_attend_split : f32 ? launch_attend_prompt_f32 : launch_attend_prompt;
    // A launch's threads are counted in 32 bits: so many workgroups of 256 threads and more (of 512 for fp32 prompts).  Whole sequences a launch.
    const int64_t blocks = call.kv * (prompt ? (rows + 127) / 128 * (f32 ? 2 : 1) : (rows + 15) / 16), at_once = kMostBlocks / blocks;
    if (call.count <= at_once) return launch(ctx, call, (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
    if (at_once < 1) return CURDKV_ERR_UNSUPPORTED;
    const int64_t bytes = f32 ? 4 : 2, queries = (int64_t)call.kv * rows;
    for (int64_t b = 0; b < call.count; b += at_once) {
        AttendCall some = call;
        some.count = std::min(at_once, call.count - b);
        some.Q = (const char*)call.Q + b * queries * kHeadDim * bytes;
        some.out = (char*)call.out + b * queries * kHeadDim * bytes;
        if (call.lse) some.lse = call.lse + b * queries;
        if (call.K) some.K = (const char*)call.K + b * call.kv * call.stride * kHeadDim * bytes;
        if (call.V) some.V = (const char*)call.V + b * call.kv * call.stride * kHeadDim * bytes;
        if (call.lengths) some.lengths = call.lengths + b;
        if (call.offsets) some.offsets = call.offsets + b * call.kv;
        some.rows = call.rows * some.count / call.count;                // (as far as the host knows)
        if (launch(ctx, some, (hipStream_t)stream) != hipSuccess) return CURDKV_ERR_HIP;
    }
    return CURDKV_OK;
}

int run_kept(curdkv_ctx* ctx, const void* Q, const void* K_kept, const void* V_kept, const uint8_t* K_scales, const uint8_t* V_scales,
             const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride,
             const int32_t* tail_lengths, int64_t count, int64_t m, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes, void* stream) {
    AttendCall c;
    const int rc = check_kept(ctx, &c, Q, K_kept, V_kept, K_scales, V_scales, offsets, total, rows, K_tail, V_tail, tail_n, tail_stride, tail_lengths, count, 1, m, scale,
                              out, lse, scratch, scratch_bytes);
    if (rc != CURDKV_OK) return rc;
    return run_attend(ctx, c, stream);
}

}  // namespace

extern "C" {

int curdkv_rotate(curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride, const int32_t* starts,
                  const int32_t* positions, const float* table, int64_t table_rows, const void* q_weight, const void* k_weight, float eps,
                  int32_t pairs, void* Q, void* K, void* V, int64_t stride, void* stream) {
    const int rc = check_rotate(ctx, qkv, count, m, row_stride, table, table_rows, q_weight, k_weight, eps, pairs, Q, K, V, stride);
    if (rc != CURDKV_OK) return rc;
    return launch_rotate(ctx, qkv, count, m, row_stride, starts, positions, nullptr, table, table_rows, q_weight, k_weight, eps, pairs == 1, Q, K, V, stride,
                         (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
}

int curdkv_attend(curdkv_ctx* ctx, const void* Q, const void* K, const void* V, int64_t count, int64_t m, int64_t n, int64_t stride,
                  const int32_t* lengths, int64_t window, int32_t n_sink, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes, void* stream) {
    const int rc = check_attend(ctx, Q, out, count, m, n, stride, scale, scratch, scratch_bytes);
    if (rc != CURDKV_OK) return rc;
    if (!K || !V || n < 1 || m > ctx->cfg.max_tokens || window < 0 || n_sink < 0 || !aligned16({K, V})) return CURDKV_ERR_INVALID_ARG;
    AttendCall c{};
    c.Q = Q, c.out = out, c.lse = lse, c.count = count;
    c.kv = ctx->cfg.kv_heads, c.group = ctx->cfg.group_size, c.m = (int)m, c.dtype = ctx->cfg.dtype, c.scale = scale;
    c.K = K, c.V = V, c.stride = stride, c.lengths = lengths, c.n = (int)n;
    c.window = window < n ? (int)window : 0, c.sinks = (int)std::min<int64_t>(n_sink, n);     // (a window of n tokens hides nothing)
    c.scratch = scratch, c.scratch_bytes = scratch_bytes;
    return run_attend(ctx, c, stream);
}

int curdkv_compact_mx(curdkv_ctx* ctx, const void* K, const void* V, int64_t n, const int32_t* indices, const int64_t* offsets, int64_t total,
                      uint8_t* K_codes, uint8_t* K_scales, uint8_t* V_codes, uint8_t* V_scales, void* stream) {
    if (!ctx || !K || !V || !offsets) return CURDKV_ERR_INVALID_ARG;
    if (!on_device_of(ctx)) return CURDKV_ERR_INVALID_ARG;
    if (n < 1 || n > ctx->cfg.max_tokens || total < 0 || total > ctx->heads * n || !aligned16({K, V, K_codes, V_codes})) return CURDKV_ERR_INVALID_ARG;
    if (total == 0) return CURDKV_OK;
    if (!indices || !K_codes || !K_scales || !V_codes || !V_scales) return CURDKV_ERR_INVALID_ARG;
    if (total > (1LL << 29)) return CURDKV_ERR_UNSUPPORTED;            // (a launch's threads are counted in 32 bits)
    return launch_compact_mx(ctx, K, V, n, indices, offsets, total, ctx->heads, K_codes, K_scales, V_codes, V_scales, (hipStream_t)stream) == hipSuccess
               ? CURDKV_OK : CURDKV_ERR_HIP;
}

int curdkv_expand_mx(curdkv_ctx* ctx, const uint8_t* codes, const uint8_t* scales, int64_t rows, void* out, void* stream) {
    if (!ctx || rows < 0) return CURDKV_ERR_INVALID_ARG;
    if (!on_device_of(ctx)) return CURDKV_ERR_INVALID_ARG;
    if (rows == 0) return CURDKV_OK;
    if (!codes || !scales || !out || !aligned16({codes, out})) return CURDKV_ERR_INVALID_ARG;
    if (rows > (1LL << 31) - 1) return CURDKV_ERR_UNSUPPORTED;         // (more than the memory holds)
    return launch_expand_mx(ctx->cfg.dtype, codes, scales, rows, out, (hipStream_t)stream) == hipSuccess ? CURDKV_OK : CURDKV_ERR_HIP;
}

int curdkv_attend_kept(curdkv_ctx* ctx, const void* Q, const void* K_kept, const void* V_kept, const int64_t* offsets, int64_t total,
                       int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride, const int32_t* tail_lengths,
                       int64_t count, int64_t m, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes, void* stream) {
    return run_kept(ctx, Q, K_kept, V_kept, nullptr, nullptr, offsets, total, rows, K_tail, V_tail, tail_n, tail_stride, tail_lengths, count, m, scale, out,
                    lse, scratch, scratch_bytes, stream);
}

int curdkv_attend_kept_mx(curdkv_ctx* ctx, const void* Q, const uint8_t* K_codes, const uint8_t* K_scales, const uint8_t* V_codes,
                          const uint8_t* V_scales, const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n,
                          int64_t tail_stride, const int32_t* tail_lengths, int64_t count, int64_t m, float scale, void* out, float* lse,
                          void* scratch, int64_t scratch_bytes, void* stream) {
    if (total > 0 && (!K_scales || !V_scales)) return CURDKV_ERR_INVALID_ARG;
    // (nothing kept: the scales are not looked at)
    return run_kept(ctx, Q, K_codes, V_codes, K_scales, V_scales, offsets, total, rows, K_tail, V_tail, tail_n, tail_stride, tail_lengths, count, m, scale,
                    out, lse, scratch, scratch_bytes, stream);
}

}  // extern "C"
