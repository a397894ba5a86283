// Products of rows in microscaled 4-bit floating point, by experts: out[m, n] = sum_k A[src(m), k] * B[g(m), n, k]
// (ftk_mx4_matmul, ftk_mx4_linear) and the sums over an expert's own rows (ftk_mx4_outer), whose
// operands are packed across the rows, so that both are products of packed rows along k.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 32 codes (16 bytes) and the block's exponent byte from every lane: lane l holds
// row l % 16 and elements 32 * (l / 16) ... of 128, which is how packed rows lie in memory.  B is the instruction's first
// operand, so that a lane ends up with four consecutive columns of one output row.  Products of 4-bit elements are
// exact; the instruction's sum of 128 was measured within 2^-24 of the sum of magnitudes.
#include "ftk_mma.h"
#include "ftk_mx4.h"

namespace ftk {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

struct MxProduct {
    const uint8_t *a_codes, *a_scales;  // packed rows, or
    const void *X;                      // dense ones
    int64_t ldx;
    int64_t N;       // rows of A
    int K;           // elements of a row
    int64_t pitch;   // blocks of 32 in a packed row (16 bytes of codes, one of scales each)
    const uint8_t *b_codes, *b_scales;
    int64_t M;       // output rows (of one expert: sums over rows)
    int F;           // output columns
    int E;
    const int32_t *offsets, *order;
    int k;
    void *out;
    int64_t ldo;
    int ntiles;      // column tiles
    int by_row;      // row tiles are numbered by their first row (few rows), else by tiles before them
};

// Expert e has the output rows [first_row(e), first_row(e + 1)); e = E stands for the rows after all of them.  Offsets are data:
// whatever they hold, the rows stay within [0, M].
__device__ __forceinline__ int64_t first_row(const MxProduct &a, int e)
{
    if (e <= 0) return 0;
    if (e > a.E || !a.offsets) return a.M;
    const int64_t o = a.offsets[e];
    return o < 0 ? 0 : o < a.M ? o : a.M;
}

// The work of a workgroup's row tile of TM rows: its rows, its expert, or nothing.
// Numbered by tiles, expert e starts at number first_row(e) / TM + e, which leaves room for its last, broken tile;
// with few rows a tile belongs to the row that it starts at.  Either way the expert is the last one whose number is
// not above the tile's: 64 lanes look at 64 of them at a time.
struct RowTile {
    int e;
    int64_t m0, end;
};
template <int TM>
__device__ __forceinline__ bool find_tile(const MxProduct &a, int64_t t, RowTile &r)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = a.E;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, e = lo + (lane + 1) * step;
        bool below = false;
        if (e <= hi) below = a.by_row ? first_row(a, e) <= t : first_row(a, e) / TM + e <= t;
        lo += __popcll(__ballot(below)) * step;
        hi = min(hi, lo + step - 1);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int64_t first = first_row(a, lo);
    r.e = lo;
    r.end = first_row(a, lo + 1);
    if (a.by_row) {
        if (t < first || (t - first) % TM) return false;
        r.m0 = t;
    } else {
        r.m0 = first + (t - (first / TM + lo)) * TM;
    }
    return r.m0 >= first && r.m0 < r.end;
}

__device__ __forceinline__ int64_t source_row(const MxProduct &a, int64_t m)
{
    int64_t s = m;
    if (a.order) {
        const int32_t o = a.order[m];
        s = o < 0 ? -1 : o / a.k;
    }
    return s < a.N ? s : -1;
}

template <typename Out>
__device__ __forceinline__ void store4(Out *o, int n, int F, float4v v)
{
    typedef Out Four __attribute__((ext_vector_type(4), aligned(sizeof(Out))));
    if (n + 4 <= F) {
        *reinterpret_cast<Four *>(o + n) = Four{(Out)v[0], (Out)v[1], (Out)v[2], (Out)v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < F) o[n + i] = (Out)v[i];
    }
}

__device__ __forceinline__ int8v frag(uint4 c) { return int8v{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}; }
__device__ __forceinline__ float4v mx_mma(uint4 b, uint32_t bs, uint4 a, uint32_t as, float4v c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(b), frag(a), c, 4, 4, 0, (int)bs, 0, (int)as);
}

// Few rows: 16 output rows by 16 * CT columns a workgroup, whose four waves share the steps of 128 elements out between
// them and add their sums up in LDS.  Operands go from memory straight to registers; a dense row is packed on
// the way, the whole block of 32 within a lane.
template <typename Src, typename Out, int CT, bool OUTER>
__global__ __launch_bounds__(256) void mx_direct_kernel(MxProduct a)
{
    constexpr bool DENSE = !std::is_same<Src, uint8_t>::value;
    __shared__ float4v part[4][CT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
    const int64_t t = blockIdx.x / a.ntiles;
    const int n0 = (int)(blockIdx.x - t * a.ntiles) * 16 * CT;
    int64_t m, end;
    int e;
    int k0 = 0, k1 = (int)(((int64_t)a.K + 127) / 128);
    if constexpr (OUTER) {
        const int64_t mt = (a.M + 15) / 16;
        e = (int)(t / mt);
        m = (t - (int64_t)e * mt) * 16 + row;
        end = a.M;
        if (a.offsets) {
            k0 = min(k1, max(0, a.offsets[e]) / 128);
            k1 = min(k1, max(0, a.offsets[e + 1]) / 128);
        }
    } else {
        RowTile r;
        if (!find_tile<16>(a, t, r)) return;
        e = r.e;
        m = r.m0 + row;
        end = r.end;
        if (e >= a.E) k1 = 0;
    }
    const int64_t src = m >= end ? -1 : OUTER ? m : source_row(a, m);
    float4v acc[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) acc[i] = float4v{0, 0, 0, 0};
    const int64_t brow = OUTER ? 0 : (int64_t)e * a.F;
    for (int s = k0 + w; s < k1; s += 4) {
        const int64_t blk = (int64_t)s * 4 + q;
        uint4 x = make_uint4(0, 0, 0, 0);
        uint32_t xs = 0;
        if (src >= 0) {
            if constexpr (DENSE) {
                const Src *p = (const Src *)a.X + src * a.ldx;
                Src v[32];
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    load8(p, blk * 32 + 8 * i, a.K, v + 8 * i);
                    top = max(top, max8(v + 8 * i));
                }
                xs = mx_scale_byte(top);
                const float f = mx_scale_float(xs);
                x = make_uint4(mx_pack8(v, f), mx_pack8(v + 8, f), mx_pack8(v + 16, f), mx_pack8(v + 24, f));
            } else {
                x = *reinterpret_cast<const uint4 *>(a.a_codes + (src * a.pitch + blk) * 16);
                xs = a.a_scales[src * a.pitch + blk];
            }
        }
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            const int64_t at = (brow + min(n0 + 16 * i + row, a.F - 1)) * a.pitch + blk;
            acc[i] = mx_mma(*reinterpret_cast<const uint4 *>(a.b_codes + at * 16), a.b_scales[at], x, xs, acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < CT; ++i) part[w][i][lane] = acc[i];
    __syncthreads();
    if (m >= end) return;
    Out *o = (Out *)a.out + (OUTER ? ((int64_t)e * a.M + m) * a.ldo : m * a.ldo);
    for (int i = w; i < CT; i += 4)
        store4(o, n0 + 16 * i + 4 * q, a.F, part[0][i][lane] + part[1][i][lane] + part[2][i][lane] + part[3][i][lane]);
}

template <typename Src, typename Out, bool OUTER>
static ftk_status launch_direct(MxProduct a, hipStream_t st)
{
    constexpr int CT = 4;
    a.ntiles = (int)ceil_div(a.F, 16 * CT);
    int64_t mtiles;
    if (OUTER) {
        mtiles = ceil_div(a.M, 16) * a.E;
    } else {
        mtiles = a.M / 16 + a.E + 1;
        a.by_row = a.M < mtiles;
        if (a.by_row) mtiles = a.M;
    }
    if (mtiles * a.ntiles > 0x7fffffffLL) {
        set_error("too many tiles: M=%lld F=%d E=%d", (long long)a.M, a.F, a.E);
        return FTK_EINVAL;
    }
    mx_direct_kernel<Src, Out, CT, OUTER><<<(unsigned)(mtiles * a.ntiles), 256, 0, st>>>(a);
    FTK_TRY_HIP(hipGetLastError());
    return FTK_OK;
}

static size_t packed_bytes(int64_t N, int D, size_t *codes)
{
    const size_t c = align_up((size_t)N * mx_padded(D) / 2, 256);
    if (codes) *codes = c;
    return c + align_up((size_t)N * mx_padded(D) / MX_BLOCK, 256);
}

static ftk_status check_product(ftk_dtype dtype, int64_t N, const void *b_codes, const void *b_scales, int64_t M, int32_t F,
                                int32_t D, int32_t E, const int32_t *offsets, const int32_t *order, int32_t k, const void *out,
                                int64_t ldo)
{
    FTK_TRY(check_mx_type(dtype));
    if (N < 0 || M < 0 || F < 1 || D < 1 || E < 1 || N > 0x7fffffffLL || M > 0x7fffffffLL || F > MX_MAX || D > MX_MAX || E > 8192 ||
        (int64_t)E * F > 0x7fffffffLL) {
        set_error("need 0 <= N, M < 2^31, 1 <= F, D <= %d, 1 <= E <= 8192, E * F < 2^31 (got N=%lld M=%lld F=%d D=%d E=%d)",
                  MX_MAX, (long long)N, (long long)M, F, D, E);
        return FTK_EINVAL;
    }
    if (!offsets && E != 1) {
        set_error("E = %d without offsets", E);
        return FTK_EINVAL;
    }
    if (order ? k < 1 : N < M) {
        set_error(order ? "k = %d with order" : "fewer rows than the output has, and no order (k = %d)", k);
        return FTK_EINVAL;
    }
    if (ldo < F) {
        set_error("row stride %lld of out is less than F = %d", (long long)ldo, F);
        return FTK_EINVAL;
    }
    if (M == 0) return FTK_OK;
    FTK_TRY(check_ptr(b_codes, 16, "b_codes"));
    FTK_TRY(check_ptr(b_scales, 4, "b_scales"));
    if (offsets) FTK_TRY(check_ptr(offsets, 4, "offsets"));
    if (order) FTK_TRY(check_ptr(order, 4, "order"));
    return check_ptr(out, dtype_size(dtype), "out");
}

}  // namespace ftk

using namespace ftk;

extern "C" {

size_t ftk_mx4_workspace_bytes(int64_t N, int32_t D, int64_t M, int32_t F)
{
    if (N < 0 || M < 0 || D < 0 || F < 0 || N > 0x7fffffffLL || D > MX_MAX) return 0;
    return packed_bytes(N, D, nullptr);
}

ftk_status ftk_mx4_matmul(ftk_dtype out_dtype, const void *a_codes, const void *a_scales, int64_t N, const void *b_codes,
                          const void *b_scales, int64_t M, int32_t F, int32_t D, int32_t E, const int32_t *offsets,
                          const int32_t *order, int32_t k, void *out, int64_t ldo, void *workspace, size_t workspace_bytes,
                          void *hip_stream)
{
    FTK_TRY(check_product(out_dtype, N, b_codes, b_scales, M, F, D, E, offsets, order, k, out, ldo));
    if (M == 0) return FTK_OK;
    if (N > 0) {
        FTK_TRY(check_ptr(a_codes, 16, "a_codes"));
        FTK_TRY(check_ptr(a_scales, 4, "a_scales"));
    }
    (void)workspace;
    (void)workspace_bytes;
    FTK_TRY(check_device());
    const MxProduct a{(const uint8_t *)a_codes, (const uint8_t *)a_scales, nullptr, 0, N, D, mx_padded(D) / MX_BLOCK,
                      (const uint8_t *)b_codes, (const uint8_t *)b_scales, M, F, E, offsets, order, k, out, ldo, 0, 0};
    return with_mx_type(out_dtype, [&](auto tag) {
        return launch_direct<uint8_t, typename decltype(tag)::type, false>(a, (hipStream_t)hip_stream);
    });
}

ftk_status ftk_mx4_linear(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *b_codes, const void *b_scales,
                          int64_t M, int32_t F, int32_t D, int32_t E, const int32_t *offsets, const int32_t *order, int32_t k,
                          void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    FTK_TRY(check_product(dtype, N, b_codes, b_scales, M, F, D, E, offsets, order, k, out, ldo));
    if (M == 0) return FTK_OK;
    if (ldx < D) {
        set_error("row stride %lld of X is less than D = %d", (long long)ldx, D);
        return FTK_EINVAL;
    }
    if (N > 0) FTK_TRY(check_ptr(X, dtype_size(dtype), "X"));
    const size_t need = packed_bytes(N, D, nullptr);
    if (need) FTK_TRY(check_workspace(workspace, workspace_bytes, need));
    FTK_TRY(check_device());
    const MxProduct a{nullptr, nullptr, X, ldx, N, D, mx_padded(D) / MX_BLOCK, (const uint8_t *)b_codes,
                      (const uint8_t *)b_scales, M, F, E, offsets, order, k, out, ldo, 0, 0};
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return launch_direct<T, T, false>(a, (hipStream_t)hip_stream);
    });
}

ftk_status ftk_mx4_outer(ftk_dtype out_dtype, const void *a_codes, const void *a_scales, const void *b_codes,
                         const void *b_scales, int64_t rows, int32_t F, int32_t D, int32_t E, const int32_t *offsets, void *out,
                         void *hip_stream)
{
    FTK_TRY(check_mx_type(out_dtype));
    if (rows < 0 || rows > 0x7fffffffLL || F < 1 || D < 1 || F > MX_MAX || D > MX_MAX || E < 1 || E > 8192) {
        set_error("need 0 <= rows < 2^31, 1 <= F, D <= %d, 1 <= E <= 8192 (got rows=%lld F=%d D=%d E=%d)", MX_MAX,
                  (long long)rows, F, D, E);
        return FTK_EINVAL;
    }
    if (!offsets && E != 1) {
        set_error("E = %d without offsets", E);
        return FTK_EINVAL;
    }
    FTK_TRY(check_ptr(out, dtype_size(out_dtype), "out"));
    if (rows > 0) {
        FTK_TRY(check_ptr(a_codes, 16, "a_codes"));
        FTK_TRY(check_ptr(a_scales, 4, "a_scales"));
        FTK_TRY(check_ptr(b_codes, 16, "b_codes"));
        FTK_TRY(check_ptr(b_scales, 4, "b_scales"));
        if (offsets) FTK_TRY(check_ptr(offsets, 4, "offsets"));
    }
    FTK_TRY(check_device());
    MxProduct a{(const uint8_t *)a_codes, (const uint8_t *)a_scales, nullptr, 0, F, (int)rows, mx_padded(rows) / MX_BLOCK,
                (const uint8_t *)b_codes, (const uint8_t *)b_scales, F, D, E, rows ? offsets : nullptr, nullptr, 1, out, D, 0, 0};
    return with_mx_type(out_dtype, [&](auto tag) {
        return launch_direct<uint8_t, typename decltype(tag)::type, true>(a, (hipStream_t)hip_stream);
    });
}

}  // extern "C"
