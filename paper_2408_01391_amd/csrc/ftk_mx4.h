// Rows in microscaled 4-bit floating point: the packed layout, and packing in registers.
#pragma once

#include <hip/hip_runtime.h>

#include "ftk_internal.h"
#include "ftk_rows.h"

namespace ftk {

constexpr int MX_BLOCK = 32;  // elements under one scale
constexpr int MX_PAD = 128;   // packed rows are whole steps of the matrix instruction
constexpr int MX_MAX = 1 << 24;  // features or rows of a product at most

static inline int64_t mx_padded(int64_t D) { return (D + MX_PAD - 1) / MX_PAD * MX_PAD; }

// Exponent byte of a block from the bits of its largest magnitude: floor(log2) - 2, not below 2^-127; the
// bits of an infinity or NaN give 255.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t max_bits)
{
    const uint32_t e = max_bits >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
// The scale as the float that the conversion instructions take: they use its exponent alone, where 0 is 2^-127.
__device__ __forceinline__ float mx_scale_float(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight elements to eight codes, the first in the lowest four bits.  v_cvt_scalef32_pk_fp4_* divides by the scale
// and rounds to the nearest even code, saturating at 6.
__device__ __forceinline__ uint32_t mx_pack8(const float *v, float scale)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
    return r;
}
__device__ __forceinline__ uint32_t mx_pack8(const __bf16 *v, float scale)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair{v[0], v[1]}, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair{v[2], v[3]}, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair{v[4], v[5]}, scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair{v[6], v[7]}, scale, 3);
    return r;
}
__device__ __forceinline__ uint32_t mx_pack8(const _Float16 *v, float scale)
{
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair{v[0], v[1]}, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair{v[2], v[3]}, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair{v[4], v[5]}, scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair{v[6], v[7]}, scale, 3);
    return r;
}

// Bits of the float magnitude.  As integers they are ordered like the magnitudes, infinities and NaN on top.
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t mag_bits(__bf16 v) { return mag_bits((float)v); }
__device__ __forceinline__ uint32_t mag_bits(_Float16 v) { return mag_bits((float)v); }

// Eight consecutive elements of a row of D, zero beyond it (i: multiple of eight).
template <typename T>
__device__ __forceinline__ void load8(const T *row, int64_t i, int64_t D, T *v)
{
    if (i + 8 <= D) {
#pragma unroll
        for (int p = 0; p < 8 / PIECE<T>; ++p) {
            const PieceOf<T> q = row_piece(row + i + p * PIECE<T>);
#pragma unroll
            for (int e = 0; e < PIECE<T>; ++e) v[p * PIECE<T> + e] = q[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i + e < D ? row[i + e] : (T)0.f;
    }
}
template <typename T>
__device__ __forceinline__ uint32_t max8(const T *v)
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, mag_bits(v[e]));
    return m;
}

// calls f(tag) for the types that packed rows are made of and products come in
template <typename F>
ftk_status with_mx_type(ftk_dtype dtype, F &&f)
{
    switch (dtype) {
    case FTK_F32: return f(TypeTag<float>{});
    case FTK_BF16: return f(TypeTag<__bf16>{});
    case FTK_F16: return f(TypeTag<_Float16>{});
    default: break;
    }
    set_error("dtype %d: 4-bit calls take FTK_F32, FTK_BF16 and FTK_F16", (int)dtype);
    return FTK_EINVAL;
}
static inline ftk_status check_mx_type(ftk_dtype dtype)
{
    return with_mx_type(dtype, [](auto) { return FTK_OK; });
}

// launches shared with the products (no checks)
ftk_status launch_mx_quantize(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int D, void *codes, void *scales,
                              hipStream_t st);

}  // namespace ftk
