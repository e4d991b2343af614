// Launchers of the kernels around a compressed cache (attend_api.hip checks the arguments).
#pragma once

#include <initializer_list>

#include "curdkv_internal.h"

namespace curdkv {

// Queries and results of one attention call, [count, m, kv * group, 128], and what is attended to.
constexpr int64_t kPastCaches = 128 << 20;     // bytes that a call moves from which its rows pass the caches (Infinity Cache: 256 MB)
constexpr int64_t kScratchCounters = 16384;     // bytes at the start of a call's scratch that are zeros between the calls

// Division of 0 .. 2^31 - 1 by a number of the host's, by a product and a shift: with 2^(s-1) < d <= 2^s and m = floor(2^32 (2^s - d) / d) + 1, n / d = (n + floor(m n / 2^32)) / 2^s.
struct Divisor {
    uint32_t d, m, s;
    Divisor() = default;
    explicit Divisor(int64_t by) : d((uint32_t)by), m(0), s(0) {
        while (((uint64_t)1 << s) < d) ++s;
        m = (uint32_t)((((((uint64_t)1 << s) - d) << 32) / d) + 1);
    }
#ifdef __HIP__
    __device__ __forceinline__ int of(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s); }
    __device__ __forceinline__ int rest(int n, int quotient) const { return n - quotient * (int)d; }
#endif
};

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
                         const int32_t* positions, const uint8_t* axis_of, const float* table, int64_t table_rows, const void* q_weight,
                         const void* k_weight, float eps, bool pairs, void* Q, void* K, void* V, int64_t stride, hipStream_t stream);
// (axis_of: host, [64], or null: one axis)

hipError_t launch_compact_mx(const curdkv_ctx* ctx, const void* K, const void* V, int64_t n, const int32_t* indices, const int64_t* offsets,
                             int64_t total, int heads, uint8_t* K_codes, uint8_t* K_scales, uint8_t* V_codes, uint8_t* V_scales, hipStream_t stream);
hipError_t launch_expand_mx(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, void* out, hipStream_t stream);

// The weight that the keys of a cache got from m tokens (curdkv_attend_weights): Q, K, stride, lengths, n, window, sinks, scale, scratch of the call.
struct WeightsCall {
    const void *Q, *K;
    const float* lse;                  // [count, kv * group, m]
    int64_t count, stride;
    int kv, group, m, n, window, sinks, dtype;
    const int32_t* lengths;
    float scale, decay;
    float* mass;                       // [count, kv, mass_stride]
    int64_t mass_stride;
    void* scratch;
    int64_t scratch_bytes;
};
hipError_t launch_weights(const curdkv_ctx* ctx, const WeightsCall& call, hipStream_t stream);

// Rows of least weight leave (curdkv_evict).
constexpr int64_t kEvictMostRows = 1 << 19;     // of a head: two bitmaps and a count of either kind lie in LDS, 16 bytes for 64 rows
struct EvictCall {
    const char *K, *V;
    const float* mass;
    const int32_t *positions, *lengths;
    int64_t count, stride, out_stride, recent;
    int kv, n, keep, sinks, dtype;
    char *K_out, *V_out;
    float* mass_out;
    int32_t *positions_out, *rows;
    bool moves;                        // the selection moves the rows itself
};
hipError_t launch_evict(const curdkv_ctx* ctx, const EvictCall& call, hipStream_t stream);

// Attention of sequences that share their kept rows (curdkv_attend_shared): in `call` count prefixes, m tokens of each of share sequences a prefix.
hipError_t launch_attend_shared(const curdkv_ctx* ctx, const AttendCall& call, int share, hipStream_t stream);

constexpr int64_t kMostBlocks = (1 << 24) - 1;     // workgroups of a launch (its threads are counted in 32 bits)

inline bool aligned16(std::initializer_list<const void*> ptrs) {
    uintptr_t all = 0;
    for (const void* p : ptrs) all |= (uintptr_t)p;
    return (all & 15u) == 0;
}

// What the attention calls have in common: sizes of the queries and of one cache array (attend_api.hip).
int check_attend(const curdkv_ctx* ctx, const void* Q, const void* out, int64_t count, int64_t m, int64_t n, int64_t stride, float scale,
                 const void* scratch, int64_t scratch_bytes);
// Kept rows and tails, checked and put into a call; `count` prefixes of `share` sequences each (curdkv_attend_kept: 1).
int check_kept(const curdkv_ctx* ctx, AttendCall* c, const void* Q, const void* K_kept, const void* V_kept, const uint8_t* K_scales, const uint8_t* V_scales,
               const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail, const void* V_tail, int64_t tail_n, int64_t tail_stride,
               const int32_t* tail_lengths, int64_t count, int64_t share, int64_t m, float scale, void* out, float* lse, void* scratch, int64_t scratch_bytes);
int check_rotate(const curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride, const float* table, int64_t table_rows,
                 const void* q_weight, const void* k_weight, float eps, int32_t pairs, const void* Q, const void* K, const void* V, int64_t stride);

// The context's device is current.
inline bool on_device_of(const curdkv_ctx* ctx) {
    int dev = -1;
    return hipGetDevice(&dev) == hipSuccess && dev == ctx->device;
}

}  // namespace curdkv
