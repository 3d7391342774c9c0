// Device helpers of the key-value cache operators.
#pragma once

#include <hip/hip_runtime.h>

#include "device.h"

namespace marlin {
namespace dev {

template <typename T>
struct Elem;

template <>
struct Elem<_Float16> {
    typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
    typedef _Float16 vec4 __attribute__((ext_vector_type(4)));
    typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
    // Two softmax weights, times kWeightUnit, as the sums of two parts (see attend.hip).  The first is rounded down from a little
    // below the weight, 2^-22 of it and half of what the second part can hold at the least, so that the second is above zero too.
    static constexpr float kWeightUnit = 32768.f;
    struct Parts {
        vec2 first, rest;
    };
    static __device__ __forceinline__ Parts part(float x, float y)
    {
        constexpr float kBelow = kWeightUnit * (1.f - 0x1p-22f), kHalf = 0x1.1p-25f;
        const vec2 first = __builtin_bit_cast(vec2, __builtin_amdgcn_cvt_pkrtz(__builtin_fmaf(x, kBelow, -kHalf), __builtin_fmaf(y, kBelow, -kHalf)));
        return {first, vec2{(_Float16)__builtin_fmaf(x, kWeightUnit, -(float)first[0]), (_Float16)__builtin_fmaf(y, kWeightUnit, -(float)first[1])}};
    }
    static __device__ __forceinline__ float4_t mfma(vec8 a, vec8 b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma(vec4 a, vec4 b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0);
    }
    // e4m3 codes as numbers, exactly: the first or the second two of a dword; eight.
    static __device__ __forceinline__ uint32_t of_two_codes(uint32_t x, bool second)
    {
        return __builtin_bit_cast(uint32_t, second ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true)
                                                   : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false));
    }
    static __device__ __forceinline__ vec8 of_codes(uint32_t x, uint32_t y)
    {
        const u32x4_t w = {of_two_codes(x, false), of_two_codes(x, true), of_two_codes(y, false), of_two_codes(y, true)};
        return __builtin_bit_cast(vec8, w);
    }
};

template <>
struct Elem<__bf16> {
    typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
    typedef __bf16 vec4 __attribute__((ext_vector_type(4)));
    typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
    static constexpr float kWeightUnit = 1.f;
    struct Parts {
        vec2 first, rest;
    };
    static __device__ __forceinline__ Parts part(float x, float y)
    {
        constexpr float kBelow = 1.f - 0x1p-22f;
        const uint32_t a = __builtin_bit_cast(uint32_t, x * kBelow), b = __builtin_bit_cast(uint32_t, y * kBelow);
        const float u = __builtin_bit_cast(float, a & 0xFFFF0000u), v = __builtin_bit_cast(float, b & 0xFFFF0000u);
        return {__builtin_bit_cast(vec2, __builtin_amdgcn_perm(b, a, 0x07060302u)), vec2{(__bf16)(x - u), (__bf16)(y - v)}};
    }
    static __device__ __forceinline__ float4_t mfma(vec8 a, vec8 b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma(vec4 a, vec4 b, float4_t c)
    {
        typedef short short4_t __attribute__((ext_vector_type(4)));
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4_t, a), __builtin_bit_cast(short4_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t of_two_codes(uint32_t x, bool second)
    {
        return __builtin_bit_cast(uint32_t, second ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true)
                                                   : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
    }
    static __device__ __forceinline__ vec8 of_codes(uint32_t x, uint32_t y)
    {
        const u32x4_t w = {of_two_codes(x, false), of_two_codes(x, true), of_two_codes(y, false), of_two_codes(y, true)};
        return __builtin_bit_cast(vec8, w);
    }
};

// N adjacent dwords, aligned to their size (three: to one).
template <int N>
__device__ __forceinline__ void load_dwords(uint32_t (&to)[N], const void *from)
{
    __builtin_memcpy(to, __builtin_assume_aligned(from, N == 3 ? 4 : 4 * N), 4 * N);
}

// The same of what is read once (see attend.hip).
template <int N>
__device__ __forceinline__ void load_dwords_once(uint32_t (&to)[N], const void *from)
{
    if constexpr (N == 3) {  // aligned to a dword only
        typedef uint32_t dword3 __attribute__((ext_vector_type(3), aligned(4)));
        const dword3 x = __builtin_nontemporal_load((const dword3 *)from);
#pragma unroll
        for (int i = 0; i < 3; ++i) to[i] = x[i];
    } else {
        typedef uint32_t dwordn __attribute__((ext_vector_type(N)));
        const dwordn x = __builtin_nontemporal_load((const dwordn *)from);
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = x[i];
    }
}

template <int N>
__device__ __forceinline__ void store_dwords(void *to, const uint32_t (&from)[N])
{
    __builtin_memcpy(__builtin_assume_aligned(to, N == 3 ? 4 : 4 * N), from, 4 * N);
}

// A word at an address that is the same in every lane and that nothing writes during the
// kernel: by the scalar cache, whose loads the vector ones do not wait for.
__device__ __forceinline__ int scalar_load(const int32_t *p)
{
    return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p;
}
__device__ __forceinline__ float scalar_load(const float *p)
{
    return *(const __attribute__((address_space(4))) float *)(uintptr_t)p;
}

// x of lane l and of lane l ^ D, D = 32 or 16, in the same order in both: an
// exchange of the wave's halves (of its odd and even 16-lane rows) between two
// registers that both hold x.
struct Pair {
    float a, b;
};
template <int D>
__device__ __forceinline__ Pair exchange(float x)
{
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto s = D == 32 ? __builtin_amdgcn_permlane32_swap(w, w, false, false) : __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const uint32_t a = s[0], b = s[1];  // named: a bit cast of a vector's element s[1] yields s[0]
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

// Over lanes l, l ^ 16, l ^ 32, l ^ 48 (the four groups of 16).
__device__ __forceinline__ float max_over_groups(float x)
{
    const Pair p = exchange<32>(x);
    const Pair q = exchange<16>(fmaxf(p.a, p.b));
    return fmaxf(q.a, q.b);
}

__device__ __forceinline__ float sum_over_groups(float x)
{
    x += __shfl_xor(x, 32);
    return x + __shfl_xor(x, 16);
}

// Inclusive sums over the lanes, by row shifts and broadcasts of a row's last lane.
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);  // row_bcast:31 into rows 2 and 3
    return x;
}

// One float of a partial result, past the L2s that are not coherent.
__device__ __forceinline__ void store_float(float *to, float x)
{
    __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// A float4 or a float of the partial results, `slot` bytes into them (the same in
// every lane) and `at` bytes further.
__device__ __forceinline__ float4_t load_slot16(__amdgpu_buffer_rsrc_t partials, int slot, int at)
{
    return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(partials, at, slot, kAuxDeviceCoherent));
}
__device__ __forceinline__ float load_slot4(__amdgpu_buffer_rsrc_t partials, int slot, int at)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(partials, at, slot, kAuxDeviceCoherent));
}

}  // namespace dev
}  // namespace marlin
