// Packing of dense rows to microscaled 4-bit floating point, along the rows or across them, and back.
//
// All three are bound by the bytes of the dense side: 17/32 of a byte is written for every element read (or
// the reverse), and the arithmetic is one conversion instruction for two elements.
#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

// Threads of both row kernels take eights of the padded rows in order, 256 at a time and MX_UNITS times a workgroup.  The
// row of a workgroup's first one is found by one wide division, what lies between by a narrow one: a wide one for every
// eight cost as much as the conversion (65536 x 2048 bf16 back: 98 us).
// (Few eights, for which there is a compute unit each: one at a time.)
constexpr int MX_UNITS = 4, MX_FEW_UNITS = 256 * 256 * 4;
struct MxUnit {
    int64_t row;
    int piece;  // eight of the row
};
template <int UNITS, typename F>
__device__ __forceinline__ void for_units(int64_t N, uint32_t pieces, F &&f)
{
    const int64_t u0 = (int64_t)blockIdx.x * (256 * UNITS), row0 = u0 / pieces;
    const uint32_t first = (uint32_t)(u0 - row0 * pieces) + threadIdx.x;
    const int64_t left = N * pieces - u0;
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        if (k * 256 + threadIdx.x >= left) break;
        const uint32_t at = first + k * 256, rows = at / pieces;
        f(MxUnit{row0 + rows, (int)(at - rows * pieces)}, u0 + k * 256 + threadIdx.x);
    }
}

// Eight elements a thread, four threads a block: the largest magnitude passes between them by two lane
// moves.  A thread's codes are one dword, so a wave writes 256 consecutive bytes.
template <typename T, int UNITS>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ X, int64_t ldx, int64_t N, int D, int pieces,
                                                          uint32_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    for_units<UNITS>(N, pieces, [&](MxUnit t, int64_t u) {  // (pieces: a multiple of 16)
        T v[8];
        load8(X + t.row * ldx, (int64_t)t.piece * 8, D, v);
        uint32_t m = max8(v);
        m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));
        m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));
        const uint32_t b = mx_scale_byte(m);
        codes[u] = mx_pack8(v, mx_scale_float(b));
        if ((t.piece & 3) == 0) scales[u >> 2] = (uint8_t)b;
    });
}

// Across the rows: a lane has the 32 rows of a block in two neighbouring columns, a wave 128 columns and two
// blocks, a workgroup 256 rows: 128 bytes of codes and eight scales of every column, brought together in LDS so that
// they leave by whole lines (written by the lanes that made them, 16 bytes at a time: 33792 x 4096 bf16 171 us).  Workgroups that
// share a line of scales run near each other on one XCD.
// Few rows and columns: half as many rows a workgroup (HALVES = 1), for twice the workgroups (30007 x 333 fp32 15.9 us with 256).
constexpr int ACROSS_COLS = 128;
template <typename T, int HALVES>
__global__ __launch_bounds__(256) void mx_quantize_across_kernel(const T *__restrict__ X, int64_t ldx, int64_t N, int D,
                                                                 int64_t nblocks, int rowgroups, uint32_t *__restrict__ codes,
                                                                 uint8_t *__restrict__ scales)
{
    // a column's dwords of codes and of scales, an odd number against bank conflicts
    constexpr int BLOCKS = 4 * HALVES, ROWS = 32 * BLOCKS, CODES = 4 * BLOCKS, LINE = CODES + HALVES + (HALVES == 2 ? 1 : 0);
    __shared__ uint32_t line[ACROSS_COLS * LINE];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t id = blockIdx.x;
    if (gridDim.x % 8 == 0) id = (id & 7) * (gridDim.x / 8) + id / 8;
    const int rg = id % rowgroups, c0 = (int)(id / rowgroups) * ACROSS_COLS;
    const int d = c0 + lane * 2;
    typedef T Pair __attribute__((ext_vector_type(2), aligned(sizeof(T))));
    const bool both = d + 1 < D;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        const int b = w * HALVES + h;
        const int64_t r0 = (int64_t)rg * ROWS + b * 32;
        T v[2][32];
        if (r0 + 32 <= N && both) {
            const T *x = X + r0 * ldx + d;
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                const Pair p = *reinterpret_cast<const Pair *>(x + r * ldx);
                v[0][r] = p[0];
                v[1][r] = p[1];
            }
        } else {
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                v[0][r] = r0 + r < N && d < D ? X[(r0 + r) * ldx + d] : (T)0.f;
                v[1][r] = r0 + r < N && both ? X[(r0 + r) * ldx + d + 1] : (T)0.f;
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = max(m, max8(&v[c][8 * i]));
            const uint32_t s = mx_scale_byte(m);
            const float f = mx_scale_float(s);
            uint32_t *l = line + (lane * 2 + c) * LINE;
#pragma unroll
            for (int i = 0; i < 4; ++i) l[b * 4 + i] = mx_pack8(&v[c][8 * i], f);
            reinterpret_cast<uint8_t *>(l + CODES)[b] = (uint8_t)s;
        }
    }
    __syncthreads();
    const int blocks = (int)(nblocks - (int64_t)rg * BLOCKS < BLOCKS ? nblocks - (int64_t)rg * BLOCKS : BLOCKS);  // 4 or 8
    for (int i = threadIdx.x; i < ACROSS_COLS * BLOCKS; i += 256) {
        const int col = i / BLOCKS, piece = i % BLOCKS;
        if (c0 + col >= D || piece >= blocks) continue;
        const uint32_t *l = line + col * LINE;
        const int64_t at = (int64_t)(c0 + col) * nblocks + (int64_t)rg * BLOCKS;
        *reinterpret_cast<uint4 *>(codes + (at + piece) * 4) = make_uint4(l[piece * 4], l[piece * 4 + 1], l[piece * 4 + 2], l[piece * 4 + 3]);
        if ((piece & 3) == 0) *reinterpret_cast<uint32_t *>(scales + at + piece) = l[CODES + (piece >> 2)];
    }
}

template <typename T, int UNITS>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                            int64_t N, int D, int pieces, T *__restrict__ out, int64_t ldo,
                                                            bool stream)
{
    typedef float pair __attribute__((ext_vector_type(2)));
    for_units<UNITS>(N, pieces, [&](MxUnit t, int64_t u) {
        const int c = t.piece * 8;
        if (c >= D) return;
        const uint32_t q = codes[u], b = scales[u >> 2];
        const float s = mx_scale_float(b);
        const pair p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 1),
                           __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 3)};
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (T)(b == 255 ? __uint_as_float(0x7fc00000u) : p[e >> 1][e & 1]);
        T *o = out + t.row * ldo + c;
        if (c + 8 <= D) {
#pragma unroll
            for (int k = 0; k < 8 / PIECE<T>; ++k) {
                PieceOf<T> w;
#pragma unroll
                for (int e = 0; e < PIECE<T>; ++e) w[e] = v[k * PIECE<T> + e];
                put_piece(o + k * PIECE<T>, w, stream);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < D) o[e] = v[e];
        }
    });
}

// calls f(units of a thread, workgroups) for a row kernel
template <typename F>
static ftk_status with_units(int64_t N, int D, F &&f)
{
    const int64_t units = N * (mx_padded(D) / 8);
    if (units <= MX_FEW_UNITS) return f(std::integral_constant<int, 1>{}, (unsigned)ceil_div(units, 256));
    const int64_t g = ceil_div(units, 256 * MX_UNITS);
    if (g > 0x7fffffffLL) {
        set_error("too many elements (N=%lld D=%d)", (long long)N, D);
        return FTK_EINVAL;
    }
    return f(std::integral_constant<int, MX_UNITS>{}, (unsigned)g);
}

ftk_status launch_mx_quantize(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int D, void *codes, void *scales,
                              hipStream_t st)
{
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return with_units(N, D, [&](auto units, unsigned grid) {
            mx_quantize_kernel<T, decltype(units)::value><<<grid, 256, 0, st>>>(
                (const T *)X, ldx, N, D, (int)(mx_padded(D) / 8), (uint32_t *)codes, (uint8_t *)scales);
            FTK_TRY_HIP(hipGetLastError());
            return FTK_OK;
        });
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
    const int64_t nblocks = mx_padded(N) / MX_BLOCK, colgroups = ceil_div(D, ACROSS_COLS);
    const bool few = ceil_div(N, 256) * colgroups < 1024;
    const int64_t rowgroups = ceil_div(N, few ? 128 : 256), wgs = rowgroups * colgroups;
    if (wgs > 0x7fffffffLL) {
        set_error("transpose: too many elements (N=%lld D=%d)", (long long)N, D);
        return FTK_EINVAL;
    }
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        const auto kernel = few ? mx_quantize_across_kernel<T, 1> : mx_quantize_across_kernel<T, 2>;
        kernel<<<(unsigned)wgs, 256, 0, st>>>((const T *)X, ldx, N, D, nblocks, (int)rowgroups, (uint32_t *)codes, (uint8_t *)scales);
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
        return with_units(N, D, [&](auto units, unsigned grid) {
            mx_dequantize_kernel<T, decltype(units)::value><<<grid, 256, 0, (hipStream_t)hip_stream>>>(
                (const uint32_t *)codes, (const uint8_t *)scales, N, D, (int)(mx_padded(D) / 8), (T *)out, ldo,
                streams_out((double)N * D * sizeof(T)));
            FTK_TRY_HIP(hipGetLastError());
            return FTK_OK;
        });
    });
}

}  // extern "C"
