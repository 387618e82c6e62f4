// page_common.h -- what the kernels of the paged 8-bit cache share: code and
// row conversions, and the host checks of their descriptors.
#pragma once

#include "fkv_hip_common.h"

namespace fkv {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

constexpr float kLargestInt8 = 127.0f;
constexpr float kLargestE4m3 = 448.0f;

// Orders what the lanes of a wave wrote before it, in LDS or memory, before what
// any of them reads after it.  (A wave's operations are performed in order: it
// keeps the compiler to that order and costs no instruction.)
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four codes of a 32-bit word as fp32.
template <bool E4M3>
__device__ __forceinline__ void codes_to_f32(uint32_t w, float (&f)[4])
{
    if (E4M3) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = (float)(int8_t)(w >> (8 * e));
    }
}

// Four fp32 values to codes of a 32-bit word: to nearest, ties to even, the
// caller's values being within the format's range or a rounding of its end.
template <bool E4M3>
__device__ __forceinline__ uint32_t f32_to_codes(const float (&f)[4])
{
    if (E4M3) {
        int w = 0;
        float g[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = fminf(fmaxf(f[e], -kLargestE4m3), kLargestE4m3);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(g[0], g[1], w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(g[2], g[3], w, true);
        return (uint32_t)w;
    }
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = (int)rintf(fminf(fmaxf(f[e], -kLargestInt8), kLargestInt8));
        w |= (uint32_t)(c & 0xff) << (8 * e);
    }
    return w;
}

// The same of values that no rounding takes past the largest code.
template <bool E4M3>
__device__ __forceinline__ uint32_t near_codes(const float (&f)[4])
{
    if (E4M3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    }
    // f + 1.5 2^23 has f, rounded to nearest with ties to even, in its low bits
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(f[e] + 12582912.0f);
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Four codes of a word times a scale, each product rounded once.  (An int8 code is
// taken as what it is: through a bias of 128, 128 times the scale of the largest
// bfloat16 rows is beyond fp32 where code times scale is not.)
template <bool E4M3>
__device__ __forceinline__ void scaled_codes(uint32_t w, float s, float* f)
{
    float c[4];
    codes_to_f32<E4M3>(w, c);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = c[e] * s;
}

// Element e of a packed pair of row elements as fp32, and back (one rounding,
// to nearest, ties to even; a NaN stays one).
__device__ __forceinline__ float row_to_f32(uint32_t pair, int e, bool bf16)
{
    const uint16_t u = (uint16_t)(pair >> (16 * e));
    if (bf16) return __uint_as_float((uint32_t)u << 16);
    return (float)__builtin_bit_cast(_Float16, u);
}

__device__ __forceinline__ uint32_t f32_to_row(float f, bool bf16)
{
    if (bf16) return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f);
    return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f);
}

__device__ __forceinline__ uint32_t f32_to_row2(float a, float b, bool bf16)
{
    return f32_to_row(a, bf16) | (f32_to_row(b, bf16) << 16);
}

inline bool page_desc_ok(const fkv_page_desc* p)
{
    return p && p->n_pages >= 1 && p->n_pages <= 0x7fffffff && p->page >= 16 && p->page <= 256 && p->page % 16 == 0 &&
           p->heads >= 1 && p->heads <= 65535 && p->d >= 16 && p->d <= 256 && p->d % 16 == 0 &&
           (p->format == FKV_PAGE_INT8 || p->format == FKV_PAGE_E4M3);
}

inline bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0 && s <= ((int64_t)1 << 40); }

inline bool row_desc_ok(const fkv_row_desc* r)
{
    return r && r->group >= 1 && stride_ok(r->stride_group) && stride_ok(r->stride_token) &&
           stride_ok(r->stride_head) && (r->type == FKV_ROW_F16 || r->type == FKV_ROW_BF16);
}

}  // namespace fkv
