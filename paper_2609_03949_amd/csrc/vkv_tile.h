// vkv_tile.h -- device helpers of the attention kernels (gfx950): direct loads
// into LDS tiles, explicit LDS operand reads, compile-time loops.
#pragma once

#include <type_traits>

#include "vkv_internal.h"

namespace vkv {

typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(1))) void gbl_void_t;
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ void wg_barrier() { asm volatile("s_barrier" ::: "memory"); }

// Compile-time loop: f(std::integral_constant<int, I>) for I = 0 .. N-1.
template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// Operand reads of the tile stages, issued as explicit LDS instructions: the
// compiler sees no LDS read of a stage, so it never makes them wait for the
// direct loads still in flight into the other stages, and the lgkmcnt waits
// before each use are explicit (lds_wait: at most N of this wave's LDS
// operations outstanding; LDS operations complete in order).  Scalar memory
// loads count in lgkmcnt too and end in any order; where a tile loop issues some
// (table entries of a paged cache), one still in flight only makes a counted wait
// longer: of the N operations that may be outstanding, fewer are LDS reads then.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
template <int OFF>
__device__ __forceinline__ bf16x8_t lds_read128(uint32_t addr) {
    bf16x8_t v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF>
__device__ __forceinline__ float lds_read32(uint32_t addr) {
    float v;
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
// transposing read: within each 16-lane group, lane j supplies the address of
// 4 consecutive 16-bit elements D[j][0..3], and lane i receives D[4e + i/4][i % 4]
// for e = 0..3
template <int OFF>
__device__ __forceinline__ i16x4_t lds_read_tr16(uint32_t addr) {
    i16x4_t v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int N, typename T0, typename T1>
__device__ __forceinline__ void lds_wait(T0& x, T1& y) {
    asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(x), "+v"(y) : "n"(N));
}
// the same, for operands of one read each
template <int N, typename T0>
__device__ __forceinline__ void lds_wait(T0& x) {
    asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(x) : "n"(N));
}

// op-reduction of x over the four 16-lane groups (lanes c, c+16, c+32, c+48),
// result in all of them: two cross-lane swaps, no LDS traffic
template <typename Op>
__device__ __forceinline__ float allreduce_groups(float x, Op op) {
    const uint32_t u = __float_as_uint(x);
    const auto r32 = __builtin_amdgcn_permlane32_swap(u, u, false, false);   // lane l ^ 32
    const float y = op(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
    const uint32_t v = __float_as_uint(y);
    const auto r16 = __builtin_amdgcn_permlane16_swap(v, v, false, false);   // lane l ^ 16
    return op(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
}

// the larger of x in lanes l and l ^ 32, in both
__device__ __forceinline__ float half_max(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ bf16x8_t join(const i16x4_t& lo, const i16x4_t& hi) {
    bf16x8_t v;
    __builtin_memcpy(&v, &lo, 8);
    __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
    return v;
}

// Products P V where some weights of a tile are masked (exactly 0) and V holds values
// that are not finite: 0 times those is not 0.  v is split into its finite values
// (the others 0) and a code of the others, +inf 1, -inf 2^7, NaN 2^14 (exact in bf16);
// the codes are summed over the keys a row sees, with weight 1, which counts each kind
// (at most 64 keys a tile), and add_nonfinite adds what they are to the finite sum.
__device__ __forceinline__ bf16x8_t split_nonfinite(bf16x8_t& v) {
    u16x8_t x = __builtin_bit_cast(u16x8_t, v), code;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint16_t m = x[j] & 0x7FFFu;
        code[j] = m < 0x7F80u ? 0 : m > 0x7F80u ? 0x4680 : (x[j] & 0x8000u) ? 0x4300 : 0x3F80;
        x[j] = m < 0x7F80u ? x[j] : 0;
    }
    v = __builtin_bit_cast(bf16x8_t, x);
    return __builtin_bit_cast(bf16x8_t, code);
}
__device__ __forceinline__ float add_nonfinite(float o, float codes) {
    const uint32_t n = (uint32_t)codes;
    if (n & 0x7Fu) o += INFINITY;
    if ((n >> 7) & 0x7Fu) o -= INFINITY;
    if (n >> 14) o = __uint_as_float(0x7FC00000u);
    return o;
}

}  // namespace vkv
