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
    bool stream;     // the result is written past the caches
    int by_row;      // row tiles are numbered by their first row (few rows), else by tiles before them
};

// Expert e has the output rows [first_row(e), first_row(e + 1)); e = E stands for the rows after all of them.  Offsets are data:
// whatever they hold, the rows stay within [0, M].
__device__ __forceinline__ int64_t first_row(const MxProduct &a, int e)
{
    if (e > a.E || !a.offsets) return e <= 0 ? 0 : a.M;
    const int64_t o = a.offsets[e];
    return o < 0 ? 0 : o < a.M ? o : a.M;
}

// The work of a workgroup's row tile of TM rows: its rows, its expert, or nothing.
// Numbered by tiles, expert e starts at number first_row(e) / TM + e, which leaves room for its last, broken tile;
// with few rows a tile belongs to the row that it starts at.  Either way the expert is the last one whose number is
// not above the tile's: 64 lanes look at 64 of them at a time.  Tiles of the first expert start at row 0; those of its rows
// that lie before `begin` are nobody's.
struct RowTile {
    int e;
    int64_t m0, begin, end;
};
template <int TM>
__device__ __forceinline__ bool find_tile(const MxProduct &a, int64_t t, RowTile &r)
{
    const int lane = threadIdx.x & 63;
    auto number = [&](int64_t first, int e) { return a.by_row ? first : first / TM + e; };
    int lo = 0, hi = a.E;
    while (hi - lo > 62) {
        const int step = (hi - lo + 63) / 64, e = lo + (lane + 1) * step;
        lo += __popcll(__ballot(e <= hi && number(first_row(a, e), e) <= t)) * step;
        hi = min(hi, lo + step - 1);
    }
    // lane i: expert lo + i, up to the end of hi (rows are less than 2^31)
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int f = (int)first_row(a, lo + lane);
    const int below = __builtin_amdgcn_readfirstlane(
        (int)__popcll(__ballot(lane > 0 && lo + lane <= hi && number((int64_t)f, lo + lane) <= t)));
    r.e = lo + below;
    r.begin = __builtin_amdgcn_readlane(f, below);
    const int64_t first = r.e ? r.begin : 0;
    r.end = __builtin_amdgcn_readlane(f, below + 1);
    if (a.by_row) {
        if (t < first || (t - first) % TM) return false;
        r.m0 = t;
    } else {
        r.m0 = first + (t - (first / TM + r.e)) * TM;
    }
    return r.m0 >= first && r.m0 < r.end;
}

// The expert with the i-th most rows, among up to 64 (else expert i).  Sums over rows take as long as an expert has rows, and
// workgroups start in order: the long ones first, so that none is left over (8 experts of 1400 to 8000 rows, 4096 x 2048
// sums each, with the packing and the rows' gradients 582 us, in the experts' own order 611).
__device__ __forceinline__ int by_size(const MxProduct &a, int i)
{
    if (!a.offsets || a.E > 64) return i;
    const int lane = threadIdx.x & 63;
    const int rows = lane < a.E ? (int)((uint32_t)a.offsets[lane + 1] - (uint32_t)a.offsets[lane]) : INT32_MIN;
    int larger = 0;
    for (int e = 0; e < a.E; ++e) {
        const int other = __builtin_amdgcn_readlane(rows, e);
        larger += other > rows || (other == rows && e < lane);
    }
    return __builtin_amdgcn_readfirstlane((int)__ffsll(__ballot(lane < a.E && larger == i)) - 1);
}

__device__ __forceinline__ int64_t source_of(const MxProduct &a, int64_t m, int32_t slot)
{
    const int64_t s = !a.order ? m : slot < 0 ? -1 : slot / a.k;
    return s < a.N ? s : -1;
}
__device__ __forceinline__ int64_t source_row(const MxProduct &a, int64_t m) { return source_of(a, m, a.order ? a.order[m] : 0); }

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

// The same onto accumulators that stay where they are, with byte BYTE of the scales.  256 of them fill the AGPRs, and the compiler,
// which may give the result other registers than the summand, would move them about.  What it would
// otherwise see to is in the text: two wait states after a vector instruction that wrote an operand.  (Before the sums are
// read, the caller waits for the last ones.)
template <int BYTE>
__device__ __forceinline__ void mx_mma_in_place(float4v &c, uint4 b, uint32_t bs, uint4 a, uint32_t as)
{
    typedef uint32_t four __attribute__((ext_vector_type(4)));
    const four x = {b.x, b.y, b.z, b.w}, y = {a.x, a.y, a.z, a.w};
    if constexpr (BYTE == 0)
        asm("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
            : "+a"(c) : "v"(x), "v"(y), "v"(bs), "v"(as));
    else
        asm("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
            : "+a"(c) : "v"(x), "v"(y), "v"(bs), "v"(as));
}
// Waits for the last of them.  The sums pass through empty statements before and behind the wait, so that no product is moved
// behind it and no look at a sum before it.
template <int MT, int NT>
__device__ __forceinline__ void mx_sums_done(float4v (&c)[MT][NT])
{
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) asm volatile("" : "+a"(c[i][j]));
    asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) asm volatile("" : "+a"(c[i][j]));
}

// Few rows: 16 output rows by 16 * CT columns a workgroup, whose WAVES waves share the steps of 128 elements out between
// them, a run each, and add their sums up in LDS.  Operands go from memory straight to registers, UNROLL steps
// at a time, all requested before the first is used: with one row the weights' way from memory is all the time there
// is.  A dense row is packed on the way, the whole block of 32 within a lane.  (One token, two matrices of 4096 x 4096: 17.8 MB in 9.6
// to 9.9 us with 32 columns and 8 waves a workgroup, 1.8 TB/s, of which the bytes alone would take 3.5; how much of the rest is
// the launch, the requests that wait for offsets and order, and the packing has not been told apart.  16 columns 11.2, 64
// columns 13.0, 16 waves 9.5.)
template <typename Src, typename Out, int CT, int WAVES, bool OUTER>
__global__ __launch_bounds__(64 * WAVES) void mx_direct_kernel(MxProduct a)
{
    constexpr bool DENSE = !std::is_same<Src, uint8_t>::value;
    constexpr int UNROLL = 4 / CT > 1 ? 4 / CT : 1;
    __shared__ float4v part[WAVES][CT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
    const int64_t t = blockIdx.x / a.ntiles;
    const int n0 = (int)(blockIdx.x - t * a.ntiles) * 16 * CT;
    int64_t m, end, src;
    int e;
    int k0 = 0, k1 = (int)(((int64_t)a.K + 127) / 128);
    if constexpr (OUTER) {
        const int64_t mt = (a.M + 15) / 16;
        e = (int)(t / mt);
        m = (t - (int64_t)e * mt) * 16 + row;
        end = a.M;
        src = m < end ? m : -1;
        if (a.offsets) {
            k0 = min(k1, max(0, a.offsets[e]) / 128);
            k1 = min(k1, max(0, a.offsets[e + 1]) / 128);
        }
    } else {
        // (numbered by rows, the tile's first row is known, and the rows of A need not wait for the expert)
        const bool early = a.by_row && a.order;
        const int32_t slot = early && t + row < a.M ? a.order[t + row] : -1;
        RowTile r;
        if (!find_tile<16>(a, t, r)) return;
        e = r.e;
        m = r.m0 + row;
        end = r.end;
        if (e >= a.E) k1 = 0;
        src = m < r.begin || m >= end ? -1 : early ? source_of(a, m, slot) : source_row(a, m);
    }
    float4v acc[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) acc[i] = float4v{0, 0, 0, 0};
    const int64_t brow = OUTER ? 0 : (int64_t)e * a.F;
    const uint8_t *bc[CT], *bs[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) {
        const int64_t at = (brow + min(n0 + 16 * i + row, a.F - 1)) * a.pitch + q;
        bc[i] = a.b_codes + at * 16;
        bs[i] = a.b_scales + at;
    }
    auto read_b = [&](int s, int i, uint4 &c, uint32_t &x) {
        c = *reinterpret_cast<const uint4 *>(bc[i] + (int64_t)s * 64);
        x = bs[i][(int64_t)s * 4];
    };
    auto read_a = [&](int s, uint4 &x, uint32_t &xs) {
        const int64_t blk = (int64_t)s * 4 + q;
        x = make_uint4(0, 0, 0, 0);
        xs = 0;
        if (src < 0) return;
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
    };
    const int run = (k1 - k0 + WAVES - 1) / WAVES, last = min(k1, k0 + (w + 1) * run);
    int s = k0 + w * run;
    for (; s + UNROLL <= last; s += UNROLL) {
        uint4 x[UNROLL], b[UNROLL][CT];
        uint32_t xs[UNROLL], bx[UNROLL][CT];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < CT; ++i) read_b(s + u, i, b[u][i], bx[u][i]);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) read_a(s + u, x[u], xs[u]);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < CT; ++i) acc[i] = mx_mma(b[u][i], bx[u][i], x[u], xs[u], acc[i]);
    }
    for (; s < last; ++s) {
        uint4 x, b[CT];
        uint32_t xs, bx[CT];
#pragma unroll
        for (int i = 0; i < CT; ++i) read_b(s, i, b[i], bx[i]);
        read_a(s, x, xs);
#pragma unroll
        for (int i = 0; i < CT; ++i) acc[i] = mx_mma(b[i], bx[i], x, xs, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < CT; ++i) part[w][i][lane] = acc[i];
    __syncthreads();
    if (m >= end) return;
    Out *o = (Out *)a.out + (OUTER ? ((int64_t)e * a.M + m) * a.ldo : m * a.ldo);
    for (int i = w; i < CT; i += WAVES) {
        float4v sum = part[0][i][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += part[v][i][lane];
        if (src < 0) sum = float4v{0, 0, 0, 0};  // (zeros times a matrix that holds NaN are not)
        store4(o, n0 + 16 * i + 4 * q, a.F, sum);
    }
}

template <typename Src, typename Out, int CT, int WAVES, bool OUTER>
static ftk_status launch_direct(MxProduct a, hipStream_t st)
{
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
    mx_direct_kernel<Src, Out, CT, WAVES, OUTER><<<(unsigned)(mtiles * a.ntiles), 64 * WAVES, 0, st>>>(a);
    FTK_TRY_HIP(hipGetLastError());
    return FTK_OK;
}

// Pieces of a line by their places before the key, and the reverse: those of a stage's first step (even ones) come first.
__device__ __forceinline__ int place_of_piece(int p) { return (p & 1) * 4 + (p >> 1); }
__device__ __forceinline__ int piece_at(int place) { return (place & 3) * 2 + (place >> 2); }

// Many rows: TM = 32 * MT rows by TN = 32 * NT columns a workgroup, a quarter of them a wave.  k goes in stages of 256
// elements, one 128-byte line of codes a row, copied straight to LDS a stage ahead of their use; scales go two
// stages (16 bytes a row) at a time.  A stage is two steps of the instruction.  Which 128 of its elements a step takes is
// free as long as both operands agree: lane quarter q takes blocks 2q and 2q + 1, so that the scales of both steps
// are one 16-bit word, out of which the instruction picks the byte.  While one step's fragments are multiplied the next
// one's are read.
//
// LDS rows are lines of eight 16-byte pieces.  Those that a stage's first step reads come first, and a row's key, half the
// lane row that reads the line, is xored into the place.  Measured at the large case below, summed over the chip: 9.4e6
// LDS cycles are lost to bank conflicts beside 2.3e7 of access; with the pieces in their own order it was 2.8e7, and the
// call took 392 us in place of 386 (one run).  The copy keeps the order of its lanes, so it is the lanes' addresses that are
// permuted, within a line.
// Column tile j of a wave has, for lane row r, column 32 * (j / 2) + 8 * (r / 4) + 4 * (j % 2) + r % 4: two
// tiles together give a lane eight consecutive columns to store.
//
// 256 x 256 sums a workgroup (MT = NT = 8), one workgroup a compute unit: 16384 x 2 rows through 16 matrices of 4096 x 4096 in
// 340 to 365 us by the box, 3.0 to 3.2 PFLOP/s; the matrix instructions alone would take 160 at the rate that power leaves them on
// such data (6.9 PFLOP/s; 9 on zeros).  The rest: copies 90, of which scales 32, writing the results 55, LDS reads 35; they
// do not hide behind the products, for a wave has its SIMD to itself and issues in order.  Two waves a SIMD (wave tiles of
// 128 x 64) took 9 % longer, two workgroups of 256 x 128 12 %, copies four steps of 64-byte lines ahead 5 %, workgroups
// that go on to their next tile while the last one's results leave 5 %.

template <int MT, int NT>
struct TileShape {
    static constexpr int TM = 32 * MT, TN = 32 * NT, ROWS = TM + TN;
    static constexpr int STAGE = ROWS * 128, SCALES = ROWS * 16;
    static constexpr int LDS = 2 * STAGE + 2 * SCALES + TM * 4;
};

template <int MT, int NT, typename Out, bool OUTER>
__global__ __launch_bounds__(256, MT* NT >= 64 ? 1 : 2) void mx_tile_kernel(MxProduct a)
{
    using S = TileShape<MT, NT>;
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    uint8_t *const sc = lds + 2 * S::STAGE;
    int *const source = reinterpret_cast<int *>(sc + 2 * S::SCALES);
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, q = lane >> 4;
    const int64_t t = blockIdx.x / a.ntiles;
    const int n0 = (int)(blockIdx.x - t * a.ntiles) * S::TN;
    int64_t m0, begin = 0, end;
    int e, k0 = 0, k1 = (int)(a.pitch / 4);
    if constexpr (OUTER) {
        const int64_t mt = (a.M + S::TM - 1) / S::TM;
        e = (int)(t / mt);
        m0 = (t - (int64_t)e * mt) * S::TM;
        e = by_size(a, e);
        end = a.M;
        if (a.offsets) {
            k0 = min(k1, max(0, a.offsets[e]) / 128);
            k1 = min(k1, max(0, a.offsets[e + 1]) / 128);
        }
    } else {
        RowTile tile;
        if (!find_tile<S::TM>(a, t, tile)) return;
        e = tile.e;
        m0 = tile.m0;
        begin = tile.begin;
        end = tile.end;
        if (e >= a.E) k1 = 0;
    }
    float4v acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = float4v{0, 0, 0, 0};
    const int wm = (w >> 1) * 16 * MT, wn = (w & 1) * 16 * NT;

    const int steps = max(0, k1 - k0), stages = (steps + 1) / 2;
    // rows of A, -1 where an output row has none
    for (int row = tid; row < S::TM; row += 256) {
        const int64_t m = m0 + row;
        source[row] = (int)(m < begin || m >= end ? -1 : OUTER ? m : source_row(a, m));
    }
    __syncthreads();
    if (steps > 0) {
        // What this lane copies: rows lane / 8 of eights of rows, one piece of each.
        const uint32_t pitch = (uint32_t)a.pitch * 16;
        const int slot = lane & 7, l8 = lane >> 3;
        const uint8_t *abase = a.a_codes + (int64_t)k0 * 64, *bbase = a.b_codes + ((int64_t)k0 * 64 + (int64_t)n0 * pitch);
        const uint8_t *const ascales = a.a_scales + k0 * 4, *bscales = a.b_scales + (k0 * 4 + (int64_t)n0 * a.pitch);
        if constexpr (!OUTER) {
            bbase += (int64_t)e * a.F * pitch;
            bscales += (int64_t)e * a.F * a.pitch;
        }
        bbase = uniform(bbase);
        const int blast = a.F - 1 - n0;
        uint32_t arow[MT], boff[NT];  // row of A; offset from the column tile's first line
#pragma unroll
        for (int i = 0; i < MT; ++i) arow[i] = (uint32_t)max(0, source[(w * MT + i) * 8 + l8]);
        // the piece of copy i of A or B
        auto piece_a = [&](int i) __attribute__((always_inline)) { return piece_at(slot ^ (l8 >> 1) ^ (i & 1) * 4); };
        auto piece_b = [&](int i) __attribute__((always_inline)) { return piece_at(slot ^ ((l8 >> 1) & 1) ^ ((w * NT + i) & 3) * 2); };
#pragma unroll
        for (int i = 0; i < NT; ++i) boff[i] = __umul24(min((w * NT + i) * 8 + l8, blast), pitch) + piece_b(i) * 16;
        const bool small = a.pitch < 16;  // all scales of a row at once, and the next row may not be there to be read
        constexpr int SN = (S::ROWS / 64 + 3) / 4;
        if (small) {
            for (int row = tid; row < S::ROWS; row += 256) {
                const int64_t at = row < S::TM ? max(0, source[row]) : min(row - S::TM, blast);
                const uint32_t *g = reinterpret_cast<const uint32_t *>((row < S::TM ? ascales : bscales) + at * a.pitch);
                for (int c = 0; c < steps; ++c) reinterpret_cast<uint32_t *>(sc + row * 16)[c] = g[c];
            }
        }
        const int64_t last = a.pitch - 16 - (int64_t)k0 * 4;  // the last 16 scales of a row
        // Copy number c of a stage (MT + NT of them).  In half a stage the line's second half lies beyond the range, maybe beyond
        // the array: the first is read twice.
        auto copy = [&](int st, int c) __attribute__((always_inline)) {
            const uint32_t to = lds0 + (st & 1) * S::STAGE;
            const bool half = 2 * st + 2 > steps;
            if (c < MT) {
                uint32_t row = arow[c];
                asm volatile("" : "+v"(row));  // (the product would be kept for all stages in two registers a row)
                const int p = half ? piece_a(c) & 3 : piece_a(c);
                to_lds16_at(abase + (int64_t)st * 128 + p * 16 + (uint64_t)row * pitch, to + (w * MT + c) * 1024);
            } else {
                const int i = c - MT;
                uint32_t o = boff[i];
                if (half) o -= (piece_b(i) & 4) * 16;
                to_lds16_from(bbase + (int64_t)st * 128, o, to + S::TM * 128 + (w * NT + i) * 1024);
            }
        };
        // the scales of stages st and st + 1
        auto copy_scales = [&](int st) __attribute__((always_inline)) {
            const int64_t o = st * 8, at = o < last ? o : last;
#pragma unroll
            for (int i = 0; i < SN; ++i) {
                const int first = (i * 4 + w) * 64, row = first + lane;
                if (first >= S::ROWS) break;
                const uint32_t src = first < S::TM ? max(0, source[min(row, S::TM - 1)]) : min(row - S::TM, blast);
                to_lds16_at((first < S::TM ? ascales : bscales) + at + (uint64_t)src * (uint32_t)a.pitch,
                            lds0 + 2 * S::STAGE + ((st >> 1) & 1) * S::SCALES + first * 16);
            }
        };
        // where a stage's scales of a row begin in its 16 bytes
        auto scale_at = [&](int st) __attribute__((always_inline)) {
            const int64_t o = (st & ~1) * 8, at = small || o < last ? o : last;
            return (int)((st & 1) * 8 + (o - at)) + ((st >> 1) & 1) * S::SCALES;
        };
        const int lrow = wm + r, lcol = wn + (r >> 2) * 8 + (r & 3), key = r >> 1;
        const uint8_t *const fa = lds + lrow * 128, *const fb = lds + (S::TM + lcol) * 128;
        const uint8_t *const sa = sc + lrow * 16, *const sb = sc + (S::TM + lcol) * 16;
        uint4 fra[MT], frb[2][NT];
        uint32_t xa[MT], xb[2][NT];
        auto read_a = [&](int at, int i) __attribute__((always_inline)) { fra[i] = *reinterpret_cast<const uint4 *>(fa + at + i * 16 * 128); };
        auto read_b = [&](int at, int j, int set) __attribute__((always_inline)) {
            frb[set][j] = *reinterpret_cast<const uint4 *>(fb + at + (j >> 1) * 32 * 128 + (j & 1) * 4 * 128);
        };
        auto read_xa = [&](int at, int i) __attribute__((always_inline)) { xa[i] = *reinterpret_cast<const uint16_t *>(sa + at + i * 16 * 16); };
        auto read_xb = [&](int at, int j, int set) __attribute__((always_inline)) {
            xb[set][j] = *reinterpret_cast<const uint16_t *>(sb + at + (j >> 1) * 32 * 16 + (j & 1) * 4 * 16);
        };
        // One step's products, row tile by row tile; behind each the next step's fragments of that number are read, the A
        // fragment into the registers just used.  BYTE: of the scales, and the set of B fragments.
        auto step = [&](auto byte, auto copies, int cst, int at, int sat) __attribute__((always_inline)) {
            constexpr int B = decltype(byte)::value, C = decltype(copies)::value;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    mx_mma_in_place<B>(acc[i][j], frb[B][j], xb[0][j], fra[i], xa[i]);
                read_a(at, i);
                if (B) read_xa(sat, i);
#pragma unroll
                for (int j = i * NT / MT; j < (i + 1) * NT / MT; ++j) {
                    read_b(at, j, 1 - B);
                    if (B) read_xb(sat, j, 1);
                }
                if constexpr (C > 0) {
#pragma unroll
                    for (int c = i * C / MT; c < (i + 1) * C / MT; ++c) copy(cst, c);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        const int whole = steps / 2;
#pragma unroll
        for (int c = 0; c < MT + NT; ++c) copy(0, c);
        if (!small) copy_scales(0);
        wait_loads<0>();
        __syncthreads();
        if (stages > 1) {
#pragma unroll
            for (int c = 0; c < MT + NT; ++c) copy(1, c);
        }
        {
            const int at = (q ^ key) * 16, sat = scale_at(0) + 2 * q;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                read_b(at, j, 0);
                read_xb(sat, j, 0);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                read_a(at, i);
                read_xa(sat, i);
            }
        }
        using Zero = std::integral_constant<int, 0>;
        using One = std::integral_constant<int, 1>;
        using All = std::integral_constant<int, MT + NT>;
        auto stage = [&](auto copies, int st) __attribute__((always_inline)) {
            step(Zero{}, Zero{}, 0, (st & 1) * S::STAGE + ((q + 4) ^ key) * 16, 0);
            // this stage is in registers and the next one has arrived, in all waves
            wait_loads<0>();
            __syncthreads();
            if constexpr (decltype(copies)::value > 0) {
                if (!small && (st & 1) == 0) copy_scales(st + 2);
            }
            // (behind the last stage this reads what is not used)
            step(One{}, copies, st + 2, ((st + 1) & 1) * S::STAGE + (q ^ key) * 16, scale_at(st + 1) + 2 * q);
#pragma unroll
            for (int j = 0; j < NT; ++j) xb[0][j] = xb[1][j];
        };
        int st = 0;
        for (; st + 2 < stages; ++st) stage(All{}, st);
        for (; st < whole; ++st) stage(Zero{}, st);
        if (steps & 1) {  // half a stage: blocks 0 to 3 of the line
            const int at = (whole & 1) * S::STAGE + (place_of_piece(q) ^ key) * 16, sat = scale_at(whole) + q;
            // (one scale a lane: a byte, at any address)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                read_b(at, j, 0);
                xb[0][j] = sb[sat + (j >> 1) * 32 * 16 + (j & 1) * 4 * 16];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                read_a(at, i);
                xa[i] = sa[sat + i * 16 * 16];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    mx_mma_in_place<0>(acc[i][j], frb[0][j], xb[0][j], fra[i], xa[i]);
        }
    }
    mx_sums_done(acc);
    typedef Out Eight __attribute__((ext_vector_type(8), aligned(sizeof(Out))));
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + wm + i * 16 + r;
        if (m >= end) continue;
        const bool held = source[wm + i * 16 + r] >= 0;
        Out *o = (Out *)a.out + (OUTER ? (int64_t)e * a.M + m : m) * a.ldo;
#pragma unroll
        for (int j = 0; j < NT; j += 2) {
            const int n = n0 + wn + (j >> 1) * 32 + q * 8;
            Eight v;
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = held ? (Out)acc[i][j + (c >> 2)][c & 3] : (Out)0.f;
            if (n + 8 <= a.F) {
                STREAM_STORE(reinterpret_cast<Eight *>(o + n), v, a.stream);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (n + c < a.F) o[n + c] = v[c];
            }
        }
    }
}

template <int MT, int NT, typename Out, bool OUTER>
static ftk_status launch_tile(MxProduct a, hipStream_t st)
{
    using S = TileShape<MT, NT>;
    a.ntiles = (int)ceil_div(a.F, S::TN);
    a.stream = streams_out((double)a.M * a.F * (OUTER ? a.E : 1) * sizeof(Out));
    int64_t mtiles = OUTER ? ceil_div(a.M, S::TM) * a.E : a.M / S::TM + a.E + 1;
    if (!OUTER) {
        a.by_row = a.M < mtiles;
        if (a.by_row) mtiles = a.M;
    }
    if (mtiles * a.ntiles > 0x7fffffffLL) {
        set_error("too many tiles: M=%lld F=%d E=%d", (long long)a.M, a.F, a.E);
        return FTK_EINVAL;
    }
    FTK_TRY(allow_lds<S::LDS>((const void *)mx_tile_kernel<MT, NT, Out, OUTER>));
    mx_tile_kernel<MT, NT, Out, OUTER><<<(unsigned)(mtiles * a.ntiles), 256, S::LDS, st>>>(a);
    FTK_TRY_HIP(hipGetLastError());
    return FTK_OK;
}

// What the tiles of a kernel take, in about a microsecond: so many of them run at once, one starts and ends in `ends` and
// takes `stage` for 256 elements.  (Whole calls with the packing, in tiles of 256 / 128 / 64 rows and columns: 16384 x 2 rows, 16 matrices
// of 4096 x 4096 393 / 439 / 608 us; 4096 x 2 rows, 8 matrices 125 / 124 / 166; 1024 x 2 rows 45 / 46 / 51; 256 x 2 rows 39 / 25 / 22; 64
// matrices of 512 x 512, 16384 x 2 rows 34 / 29 / 31.)
static double tile_cost(const MxProduct &a, bool outer, int side, int at_once, double ends, double stage)
{
    // half of the experts with rows leave a broken tile more
    const int64_t rows = outer ? ceil_div(a.M, side) * a.E : a.M / side + (a.M < a.E ? a.M : (a.E + 1) / 2);
    const double stages = (double)a.K / (outer ? a.E : 1) / 256;
    return (double)ceil_div(rows * ceil_div(a.F, side), at_once) * (ends + stages * stage);
}

template <typename Out, bool OUTER>
static ftk_status launch_packed(const MxProduct &a, hipStream_t st)
{
    // offsets within a column tile are 32 bits wide
    if (a.N == 0 || a.pitch >= 1 << 20) return launch_direct<uint8_t, Out, 4, 4, OUTER>(a, st);
    const double large = tile_cost(a, OUTER, 256, 256, 11, 1.75), middle = tile_cost(a, OUTER, 128, 512, 6, 1.27),
                 small = tile_cost(a, OUTER, 64, 1024, 5, 0.75);
    if (large <= middle && large <= small) return launch_tile<8, 8, Out, OUTER>(a, st);
    return middle <= small ? launch_tile<4, 4, Out, OUTER>(a, st) : launch_tile<2, 2, Out, OUTER>(a, st);
}

// Whether dense rows are packed by every workgroup that needs them rather than once beforehand, in a launch of its own.  (Whole call,
// matrices of 4096 x 4096, with / without: 2 rows 12.8 / 17.5 us, 8 rows of 8 experts 18.1 / 17.8, 16 rows 25.1 / 17.6, of 4 experts 16.1 /
// 17.5, of 2 12.9 / 17.5; 32 rows of 8 29.8 / 17.5.)
static bool few_rows(int64_t M, int E) { return M <= 8 || (M <= 16 && E <= 4); }

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

int64_t ftk_mx4_workspace_bytes(int64_t N, int32_t D, int64_t M, int32_t E)
{
    if (N < 0 || M < 0 || D < 1 || E < 1 || N > 0x7fffffffLL || M > 0x7fffffffLL || D > MX_MAX) {
        set_error("need 0 <= N, M < 2^31, 1 <= D <= %d, E >= 1 (got N=%lld M=%lld D=%d E=%d)", MX_MAX, (long long)N, (long long)M, D,
                  E);
        return -1;
    }
    return N == 0 || few_rows(M, E) ? 0 : (int64_t)packed_bytes(N, D, nullptr);
}

ftk_status ftk_mx4_matmul(ftk_dtype out_dtype, const void *a_codes, const void *a_scales, int64_t N, const void *b_codes,
                          const void *b_scales, int64_t M, int32_t F, int32_t D, int32_t E, const int32_t *offsets,
                          const int32_t *order, int32_t k, void *out, int64_t ldo, void *hip_stream)
{
    FTK_TRY(check_product(out_dtype, N, b_codes, b_scales, M, F, D, E, offsets, order, k, out, ldo));
    if (M == 0) return FTK_OK;
    if (N > 0) {
        FTK_TRY(check_ptr(a_codes, 16, "a_codes"));
        FTK_TRY(check_ptr(a_scales, 4, "a_scales"));
    }
    FTK_TRY(check_device());
    const MxProduct a{(const uint8_t *)a_codes, (const uint8_t *)a_scales, nullptr, 0, N, D, mx_padded(D) / MX_BLOCK,
                      (const uint8_t *)b_codes, (const uint8_t *)b_scales, M, F, E, offsets, order, k, out, ldo, 0, false, 0};
    return with_mx_type(out_dtype, [&](auto tag) {
        return launch_packed<typename decltype(tag)::type, false>(a, (hipStream_t)hip_stream);
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
    const bool few = N == 0 || few_rows(M, E);
    if (!few) FTK_TRY(check_workspace(workspace, workspace_bytes, packed_bytes(N, D, nullptr)));
    FTK_TRY(check_device());
    hipStream_t st = (hipStream_t)hip_stream;
    MxProduct a{nullptr, nullptr, X, ldx, N, D, mx_padded(D) / MX_BLOCK, (const uint8_t *)b_codes,
                (const uint8_t *)b_scales, M, F, E, offsets, order, k, out, ldo, 0, false, 0};
    if (!few) {
        size_t codes = 0;
        packed_bytes(N, D, &codes);
        uint8_t *p = (uint8_t *)workspace;
        FTK_TRY(launch_mx_quantize(dtype, X, ldx, N, D, p, p + codes, st));
        a.a_codes = p;
        a.a_scales = p + codes;
    }
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return few ? launch_direct<T, T, 2, 8, false>(a, st) : launch_packed<T, false>(a, st);
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
                (const uint8_t *)b_codes, (const uint8_t *)b_scales, F, D, E, rows ? offsets : nullptr, nullptr, 1, out, D, 0, false, 0};
    return with_mx_type(out_dtype, [&](auto tag) {
        return launch_packed<typename decltype(tag)::type, true>(a, (hipStream_t)hip_stream);
    });
}

}  // extern "C"
