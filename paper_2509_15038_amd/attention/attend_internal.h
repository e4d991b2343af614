// Launchers of the kernels around a compressed cache (attend_api.hip checks the arguments).
#pragma once

#include "curdkv_internal.h"

namespace curdkv {

// Queries and results of one attention call, [count, m, kv * group, 128], and what is attended to.
constexpr int64_t kPastCaches = 128 << 20;     // bytes that a call moves from which its rows pass the caches (Infinity Cache: 256 MB)
constexpr int64_t kScratchCounters = 16384;     // bytes at the start of a call's scratch that are zeros between the calls

struct AttendCall {
    const void* Q;
    void* out;
    float* lse;                        // [count, kv * group, m] or nullptr
    int64_t count;
    int kv, group, m;
    int dtype;                         // CURDKV_DTYPE_* of Q, out and the cache
    float scale;
    // the cache, or the tokens since: [count, kv, stride, 128], the first lengths[b] rows (n where lengths is null, and at most n)
    const void *K, *V;
    int64_t stride;
    const int32_t* lengths;
    int n, window, sinks;
    // kept rows in front of them, seen by every token: rows offsets[i] .. offsets[i + 1] - 1 of a packed array for head i; null: none
    const int64_t* offsets;
    const void *K_kept, *V_kept;       // storage type, or codes of 4 bits where K_scales is given
    const uint8_t *K_scales, *V_scales;
    int64_t total, rows;               // rows of the arrays; of them this call's heads'
    void* scratch;                     // for partial results; null or too small: heads are shared out less
    int64_t scratch_bytes;
};

hipError_t launch_attend_split(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream);
hipError_t launch_attend_prompt(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream);     // bf16; kept rows not in 4 bits
hipError_t launch_attend_prompt_f32(const curdkv_ctx* ctx, const AttendCall& call, hipStream_t stream);

hipError_t launch_rotate(const curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride, const int32_t* starts,
                         const int32_t* positions, const float* table, int64_t table_rows, const void* q_weight, const void* k_weight,
                         float eps, bool pairs, void* Q, void* K, void* V, int64_t stride, hipStream_t stream);

hipError_t launch_compact_mx(const curdkv_ctx* ctx, const void* K, const void* V, int64_t n, const int32_t* indices, const int64_t* offsets,
                             int64_t total, int heads, uint8_t* K_codes, uint8_t* K_scales, uint8_t* V_codes, uint8_t* V_scales, hipStream_t stream);
hipError_t launch_expand_mx(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, void* out, hipStream_t stream);

// The context's device is current.
inline bool on_device_of(const curdkv_ctx* ctx) {
    int dev = -1;
    return hipGetDevice(&dev) == hipSuccess && dev == ctx->device;
}

}  // namespace curdkv
