// Rows of the cache in 4 bits (the open microscaling format): blocks of 32 channels share a power of two 2^e, stored as e + 127,
//     e = floor(log2(largest magnitude)) - 2, at least -127,
// and a channel x is held as the nearest to x 2^-e of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (ties to the even code, beyond 6
// to 6).  A block that holds an infinity or NaN has the scale 255 and stands for NaN.  64 bytes of codes, channel 2 i in the low
// half of byte i, and 4 scales a row: 68 bytes instead of 256 (bf16) or 512.
//
// compact_mx_kernel is the gather of compact_kernels.hip with that at its end: HBM-bound, a row read whole by 16 (32) lanes of 16
// bytes, K and V by different workgroups.  Four (eight) neighbouring lanes hold a block: two (three) DPP exchanges find its
// largest magnitude, on the bits, where NaN counts as larger than all.  All steps are exact but the rounding to a code.
// Measured: 3276 of 32768 rows of 256 heads gathered and expanded again (1090 MB) 180 to 185 us in three launches, 5.9 to 6.1 TB/s; of 8 heads 12.4 us, three
// launches at their shortest.  In fp32 (1950 MB) 523 us, 3.7 TB/s: stores past the caches in half lines, as in rotate_kernel.hip.

#include "attend_device.h"
#include "attend_internal.h"

namespace curdkv {
namespace {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }

// The head that owns packed row p: the last one whose rows begin at or before it.  64 offsets at a time, one a lane.  (Offsets out of order lead to a wrong
// head, never outside the cache.)
__device__ __forceinline__ int head_of_row(const int64_t* offsets, int heads, int64_t p) {
    const int lane = threadIdx.x & 63;
    int low = 0, span = heads;                                   // it lies in [low, low + span)
    while (span > 1) {
        const int step = (span + 63) / 64, i = lane * step;
        const uint64_t before = __ballot(i < span && offsets[low + min(i, span - 1)] <= p);
        const int at = before ? 63 - __builtin_clzll(before) : 0;
        low += at * step;
        span = min(step, span - at * step);
    }
    return low;
}

// ROWS a thread, all their loads in flight together.  (What is written stays in the caches, where the next call finds it: past them, gather and expansion of
// 256 x 3276 rows one after the other take 194 us instead of 184.)
template <bool BF16, int ROWS>
__global__ __launch_bounds__(256) void compact_mx_kernel(const u32x4a* __restrict__ K, const u32x4a* __restrict__ V, int64_t n,
                                                         const int32_t* __restrict__ indices, const int64_t* __restrict__ offsets,
                                                         int64_t total, int heads,
                                                         uint8_t* __restrict__ K_codes, uint8_t* __restrict__ K_scales,
                                                         uint8_t* __restrict__ V_codes, uint8_t* __restrict__ V_scales) {
    constexpr int kLanes = BF16 ? 16 : 32, kStep = 256 / kLanes, kValues = BF16 ? 8 : 4;
    const int c = threadIdx.x % kLanes;
    const int64_t p0 = (int64_t)blockIdx.x * (kStep * ROWS), p = p0 + threadIdx.x / kLanes;
    int32_t index[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) index[r] = indices[min(p + r * kStep, total - 1)];
    int h = head_of_row(offsets, heads, p0);
    int64_t head_end = h + 1 < heads ? offsets[h + 1] : total;
    bool ok[ROWS];
    u32x4a raw[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t at = p + r * kStep;
        while (head_end <= at && h + 1 < heads) {
            ++h;
            head_end = h + 1 < heads ? offsets[h + 1] : total;
        }
        ok[r] = at < total && index[r] >= 0 && index[r] < n;    // never read outside the cache
        raw[r] = __builtin_nontemporal_load((blockIdx.y ? V : K) + ((size_t)h * n + (ok[r] ? index[r] : 0)) * kLanes + c);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float x[kValues];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < kValues; ++i) {
            const uint32_t bits = BF16 ? (i % 2 ? raw[r][i / 2] & 0xFFFF0000u : raw[r][i / 2] << 16) : raw[r][i % 4];
            x[i] = __uint_as_float(bits);
            most = max(most, bits & 0x7FFFFFFFu);
        }
        most = max(most, dpp<0xB1>(most));                      // quad_perm xor 1, xor 2
        most = max(most, dpp<0x4E>(most));
        if (!BF16) most = max(most, dpp<0x141>(most));          // mirror of eight lanes
        const uint32_t field = most >> 23, e = field < 2 ? 0 : field - 2;      // e + 127
        const bool finite = field < 255;
        const float up = __uint_as_float((254u - e) << 23);     // 2^-e, exact
        uint32_t codes = 0;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0] * up, x[1] * up, 1.f, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2] * up, x[3] * up, 1.f, 1);
        if (BF16) {
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[kValues - 4] * up, x[kValues - 3] * up, 1.f, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[kValues - 2] * up, x[kValues - 1] * up, 1.f, 3);
        }
        if (!finite) codes = 0;
        if (!ok[r]) continue;
        const int64_t at = p + r * kStep;
        uint8_t* to = (blockIdx.y ? V_codes : K_codes) + at * 64;
        if (BF16) ((uint32_t*)to)[c] = codes;
        else ((uint16_t*)to)[c] = (uint16_t)codes;
        if (c % (kLanes / 4) == 0) (blockIdx.y ? V_scales : K_scales)[at * 4 + c / (kLanes / 4)] = finite ? (uint8_t)e : 255;
    }
}

// What codes and scales stand for, 8 channels a thread.  PAST: what is written passes the caches (two of 838656 rows 104 us, 82 so).
template <bool PAST, class T>
__device__ __forceinline__ void put(T x, T* to) {
    if (PAST) __builtin_nontemporal_store(x, to);
    else *to = x;
}
template <bool BF16, bool PAST>
__global__ __launch_bounds__(256) void expand_mx_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t pieces,
                                                        void* __restrict__ out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const uint32_t code = codes[i], e = scales[i / 4];
    const float unit = __uint_as_float(e << 23);           // (the conversion takes the exponent alone: 0 is 2^-127, 255 makes NaN of every code)
    float x[8];
    *(f32x2a*)(x + 0) = __builtin_bit_cast(f32x2a, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 0));
    *(f32x2a*)(x + 2) = __builtin_bit_cast(f32x2a, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 1));
    *(f32x2a*)(x + 4) = __builtin_bit_cast(f32x2a, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 2));
    *(f32x2a*)(x + 6) = __builtin_bit_cast(f32x2a, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 3));
    if (BF16) {
        put<PAST>((u32x4a){pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}, (u32x4a*)out + i);
    } else {
        put<PAST>((f32x4a){x[0], x[1], x[2], x[3]}, (f32x4a*)out + 2 * i);
        put<PAST>((f32x4a){x[4], x[5], x[6], x[7]}, (f32x4a*)out + 2 * i + 1);
    }
}

}  // namespace

hipError_t launch_compact_mx(const curdkv_ctx* ctx, const void* K, const void* V, int64_t n, const int32_t* indices, const int64_t* offsets,
                             int64_t total, int heads, uint8_t* K_codes, uint8_t* K_scales, uint8_t* V_codes, uint8_t* V_scales, hipStream_t stream) {
    const auto launch = [&](auto kernel, int rows) {
        kernel<<<dim3((unsigned)((total + rows - 1) / rows), 2), 256, 0, stream>>>((const u32x4a*)K, (const u32x4a*)V, n, indices, offsets, total,
                                                                                  heads, K_codes, K_scales, V_codes, V_scales);
    };
    // Four rows a thread where that leaves every unit eight workgroups (256 x 3276 rows: 104 us with one, 83 with four).
    const bool bf16 = ctx->cfg.dtype == CURDKV_DTYPE_BF16, many = total >= 256 * (int64_t)ctx->num_cu;
    if (bf16) many ? launch(compact_mx_kernel<true, 4>, 64) : launch(compact_mx_kernel<true, 1>, 16);
    else many ? launch(compact_mx_kernel<false, 4>, 32) : launch(compact_mx_kernel<false, 1>, 8);
    return hipGetLastError();
}

hipError_t launch_expand_mx(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, void* out, hipStream_t stream) {
    const bool bf16 = dtype == CURDKV_DTYPE_BF16;
    // (a launch's threads are counted in 32 bits: 2^27 rows each)
    const auto launch = [&](auto kernel) {
        for (int64_t first = 0; first < rows; first += 1 << 27) {
            const int64_t pieces = (rows - first < 1 << 27 ? rows - first : 1 << 27) * 16;
            kernel<<<(unsigned)((pieces + 255) / 256), 256, 0, stream>>>((const uint32_t*)(codes + first * 64), scales + first * 4, pieces,
                                                                         (char*)out + first * (bf16 ? 256 : 512));
        }
    };
    if (rows * ((bf16 ? 256 : 512) + 68) > kPastCaches) bf16 ? launch(expand_mx_kernel<true, true>) : launch(expand_mx_kernel<false, true>);
    else bf16 ? launch(expand_mx_kernel<true, false>) : launch(expand_mx_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace curdkv
