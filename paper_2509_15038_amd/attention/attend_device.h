// Attention over a cache: what the kernels share.  Notation, for one KV head: its `group` query heads and m tokens make
// rows R = token * group + head of the products' other side; token t of m stands at position p(t) = length - m + t.
#pragma once

#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "curdkv_internal.h"

// (a lambda of a kernel's that is not inlined would leave what it refers to in memory)
#define ALWAYS_INLINE __attribute__((always_inline))

namespace curdkv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4a __attribute__((ext_vector_type(4)));
typedef float f32x2a __attribute__((ext_vector_type(2)));
typedef float f32x4a __attribute__((ext_vector_type(4)));
typedef float f32x16a __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2a __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8a __attribute__((ext_vector_type(8)));

constexpr float kLn2 = 0.693147180559945309f;
// The reference of a row that has met no score yet, or none but -infinity (a hidden key's, or an infinite key's): exp2(-infinity - kNoScore) is the weight 0 that such
// a key has, where -infinity in its place would make NaN of the difference.
// A row is empty where its weights' sum is 0: the largest key weighs something, and a NaN among the scores, which maxima pass over, makes NaN of the sum.
constexpr float kNoScore = -FLT_MAX;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2a{a, b}), bf16x2a));
}

// max / sum over the four lanes l, l^16, l^32, l^48
__device__ __forceinline__ float quarters_max(float x) {
    u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float quarters_sum(float x) {
    u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r.x) + __uint_as_float(r.y);
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// The rows of a cache that some token of tokens t0 .. t1 (of the m new ones) sees: [0, first) and [low, high).
struct Seen {
    int first, low, high;
    int p0, p1;                        // positions of t0 and t1
};
__device__ __forceinline__ Seen seen_rows(int length, int m, int t0, int t1, int window, int sinks) {
    Seen s;
    s.p0 = length - m + t0;
    s.p1 = length - m + t1;
    s.high = max(0, s.p1 + 1);
    s.low = window > 0 && (int64_t)s.p0 - window + 1 > 0 ? min(s.p0 - window + 1, s.high) : 0;
    s.first = min(sinks, s.low);
    return s;
}
__device__ __forceinline__ bool sees(int p, int j, int window, int sinks) {
    return j <= p && (window <= 0 || p - j < window || j < sinks);
}

// sums and maxima of a lane's half wave with the other
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
// A value that is the same in all lanes, where the compiler does not see it.
__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32);
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

}  // namespace curdkv
