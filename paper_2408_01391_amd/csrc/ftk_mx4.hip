// Packing of dense rows to microscaled 4-bit floating point, along the rows or across them, and back.
//
// All three are bound by the bytes of the dense side: 17/32 of a byte is written for every element read (or
// the reverse), and the arithmetic is one conversion instruction for two elements.
#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

// Eight elements a thread, four threads a block: the largest magnitude passes between them by two lane
// moves.  A thread's codes are one dword, so a wave writes 256 consecutive bytes.
template <typename T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ X, int64_t ldx, int64_t N, int D, int pieces,
                                                          uint32_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const int64_t total = N * pieces;  // pieces: eights of a padded row, a multiple of 16
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / pieces;
        const int c = (int)(u - row * pieces);
        T v[8];
        load8(X + row * ldx, (int64_t)c * 8, D, v);
        uint32_t m = max8(v);
        m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));
        m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));
        const uint32_t b = mx_scale_byte(m);
        codes[u] = mx_pack8(v, mx_scale_float(b));
        if ((c & 3) == 0) scales[u >> 2] = (uint8_t)b;
    }
}

// Across the rows: a lane has the 32 rows of a block in two neighbouring columns, a wave 128 columns.
// Workgroup: four blocks (128 rows), the 64 bytes of codes and four scales that a column has of them.
template <typename T>
__global__ __launch_bounds__(256) void mx_quantize_across_kernel(const T *__restrict__ X, int64_t ldx, int64_t N, int D,
                                                                 int64_t nblocks, uint4 *__restrict__ codes,
                                                                 uint8_t *__restrict__ scales)
{
    const int lane = threadIdx.x & 63;
    const int64_t blk = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);  // of 32 rows; nblocks is a multiple of 4
    const int d = ((int)blockIdx.y * 64 + lane) * 2;
    if (d >= D) return;
    typedef T Pair __attribute__((ext_vector_type(2), aligned(sizeof(T))));
    const bool both = d + 1 < D;
    T v[2][32];
    const int64_t r0 = blk * 32;
#pragma unroll
    for (int r = 0; r < 32; ++r) {
        v[0][r] = v[1][r] = (T)0.f;
        if (r0 + r < N) {
            const T *x = X + (r0 + r) * ldx + d;
            if (both) {
                const Pair p = *reinterpret_cast<const Pair *>(x);
                v[0][r] = p[0];
                v[1][r] = p[1];
            } else {
                v[0][r] = *x;
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        if (c && !both) break;
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max8(&v[c][8 * i]));
        const uint32_t b = mx_scale_byte(m);
        const float s = mx_scale_float(b);
        codes[(int64_t)(d + c) * nblocks + blk] =
            make_uint4(mx_pack8(&v[c][0], s), mx_pack8(&v[c][8], s), mx_pack8(&v[c][16], s), mx_pack8(&v[c][24], s));
        scales[(int64_t)(d + c) * nblocks + blk] = (uint8_t)b;
    }
}

__device__ __forceinline__ float mx_value(uint32_t code, uint32_t byte)
{
    // magnitude by its two bits of exponent and one of mantissa: twice it is 0, 1, 2, 3, 4, 6, 8, 12
    const uint32_t i = code & 7;
    const float twice = i < 2 ? (float)i : (float)((2 + (i & 1)) << ((i >> 1) - 1));
    const float v = ldexpf(twice, (int)byte - 128);
    return byte == 255 ? __uint_as_float(0x7fc00000u) : code & 8 ? -v : v;
}

template <typename T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                            int64_t N, int D, int pieces, T *__restrict__ out, int64_t ldo)
{
    const int64_t total = N * pieces;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / pieces;
        const int c = (int)(u - row * pieces) * 8;
        if (c >= D) continue;
        const uint32_t q = codes[u], b = scales[u >> 2];
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (T)mx_value(q >> (4 * e), b);
        T *o = out + row * ldo + c;
        if (c + 8 <= D) {
#pragma unroll
            for (int p = 0; p < 8 / PIECE<T>; ++p) {
                PieceOf<T> w;
#pragma unroll
                for (int e = 0; e < PIECE<T>; ++e) w[e] = v[p * PIECE<T> + e];
                put_piece(o + p * PIECE<T>, w);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < D) o[e] = v[e];
        }
    }
}

static int mx_grid(int64_t threads)
{
    const int64_t g = ceil_div(threads, 256);
    return (int)(g < 65536 ? g : 65536);
}

ftk_status launch_mx_quantize(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int D, void *codes, void *scales,
                              hipStream_t st)
{
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        const int pieces = (int)(mx_padded(D) / 8);
        mx_quantize_kernel<T><<<mx_grid(N * pieces), 256, 0, st>>>((const T *)X, ldx, N, D, pieces, (uint32_t *)codes,
                                                                   (uint8_t *)scales);
        FTK_TRY_HIP(hipGetLastError());
        return FTK_OK;
    });
}

static ftk_status check_mx(ftk_dtype dtype, const void *X, int64_t ld, int64_t N, int32_t D, const void *codes,
                           const void *scales, const char *name)
{
    FTK_TRY(check_mx_type(dtype));
    if (N < 0 || N > 0x7fffffffLL || D < 1 || D > MX_MAX) {
        set_error("need 0 <= N < 2^31, 1 <= D <= %d (got N=%lld D=%d)", MX_MAX, (long long)N, D);
        return FTK_EINVAL;
    }
    if (ld < D) {
        set_error("row stride %lld of %s is less than D = %d", (long long)ld, name, D);
        return FTK_EINVAL;
    }
    if (N == 0) return FTK_OK;
    FTK_TRY(check_ptr(X, dtype_size(dtype), name));
    FTK_TRY(check_ptr(codes, 16, "codes"));
    FTK_TRY(check_ptr(scales, 4, "scales"));
    return check_device();
}

}  // namespace ftk

using namespace ftk;

extern "C" {

ftk_status ftk_mx4_quantize(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int32_t D, int32_t transpose, void *codes,
                            void *scales, void *hip_stream)
{
    FTK_TRY(check_mx(dtype, X, ldx, N, D, codes, scales, "X"));
    if (N == 0) return FTK_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!transpose) return launch_mx_quantize(dtype, X, ldx, N, D, codes, scales, st);
    const int64_t nblocks = mx_padded(N) / MX_BLOCK, wgs = nblocks / 4;
    if (ceil_div(D, 128) > 65535) {
        set_error("transpose: D = %d is too large (at most %d)", D, 128 * 65535);
        return FTK_EINVAL;
    }
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        mx_quantize_across_kernel<T><<<dim3((unsigned)wgs, (unsigned)ceil_div(D, 128)), 256, 0, st>>>(
            (const T *)X, ldx, N, D, nblocks, (uint4 *)codes, (uint8_t *)scales);
        FTK_TRY_HIP(hipGetLastError());
        return FTK_OK;
    });
}

ftk_status ftk_mx4_dequantize(ftk_dtype dtype, const void *codes, const void *scales, int64_t N, int32_t D, void *out,
                              int64_t ldo, void *hip_stream)
{
    FTK_TRY(check_mx(dtype, out, ldo, N, D, codes, scales, "out"));
    if (N == 0) return FTK_OK;
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        const int pieces = (int)(mx_padded(D) / 8);
        mx_dequantize_kernel<T><<<mx_grid(N * pieces), 256, 0, (hipStream_t)hip_stream>>>(
            (const uint32_t *)codes, (const uint8_t *)scales, N, D, pieces, (T *)out, ldo);
        FTK_TRY_HIP(hipGetLastError());
        return FTK_OK;
    });
}

}  // extern "C"
